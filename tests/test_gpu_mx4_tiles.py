"""The products at MX4 weights in every tile that their rule takes, against the float64
oracle: odd and even numbers of k-steps, ragged experts, column tiles past the matrix, more
tiles than workgroups.  Bounds as in test_gpu_mx4.py."""
import functools

import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case, dev, host
from oracle import mx4
from oracle.numerics import round_bf16
from test_gpu_mx4 import DT, _bound, _ffn_check, _ffn_inputs, _i32, _mx4, _routing

pytestmark = pytest.mark.gpu

PRODUCTS = [   # rows and columns of the tiles; T, k, E, dead, N, K
    ((32, 64), 90, 1, 4, 1, 128, 576), ((64, 128), 1500, 2, 16, 3, 1088, 704),
    ((128, 128), 6300, 1, 2, 0, 1024, 320), ((128, 128), 2100, 3, 3, 1, 1088, 192),
    # 3, 3, 4, 5, 5 steps of 256 columns; 9 and more of 64
    ((128, 256), 8100, 1, 20, 0, 2048, 576), ((128, 256), 1100, 8, 20, 3, 1984, 640),
    ((128, 256), 4100, 2, 19, 0, 2112, 1024), ((128, 256), 8500, 1, 20, 5, 2048, 1216),
    ((128, 256), 33000, 1, 80, 9, 448, 1088),
    ((256, 256), 4300, 2, 2, 0, 7104, 576), ((256, 256), 16500, 2, 3, 0, 1984, 640),
    ((256, 256), 16500, 1, 6, 1, 4096, 1024), ((256, 256), 70000, 1, 1, 0, 832, 1216),
    ((256, 256), 70000, 1, 5, 2, 832, 832)]


@functools.lru_cache(1)     # (shared by the types of one size)
def _operands(T, k, E, dead, N, K):
    g = np.random.default_rng(T + N + K)
    routing = _routing(g, T, k, E, dead, skew=1.0)
    x = round_bf16(g.normal(size=(T, K)))
    return (*routing, x, mx4.quantize(g.normal(size=(E - dead, N, K)) * 0.05), mx4.quantize(x))


@functools.lru_cache(1)
def _reference(T, k, E, dead, N, K, act):
    row_src, offsets, emap, x, qw, qx = _operands(T, k, E, dead, N, K)
    xv = mx4.dequantize(*qx) if act == 4 else x
    return mx4.grouped_product(xv[row_src // k], mx4.dequantize(*qw), offsets, emap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("tile,T,k,E,dead,N,K", PRODUCTS)
def test_product(tile, T, k, E, dead, N, K, act, dtype):
    case(f"mx4 product tile={tile} T={T} k={k} E={E} dead={dead} N={N} K={K} act={act} {dtype}")
    assert laep.laep_mx4_product_tile(T * k, E, N, K, act) == tile
    row_src, offsets, emap, x, qw, qx = _operands(T, k, E, dead, N, K)
    ref, mag = _reference(T, k, E, dead, N, K, act)
    live = ~np.isnan(ref)            # (the oracle's mark: rows of experts without a slot)
    out = torch.full((T * k, N), 7.0, dtype=DT[dtype], device="cuda")
    args = (_mx4(qx) if act == 4 else dev(x, torch.bfloat16), _mx4(qw), _i32(offsets))
    kw = dict(row_src=_i32(row_src), k=k, expert_map=_i32(emap), dtype=DT[dtype])
    laep.moe_mx4_grouped_product(*args, out=out, **kw)
    got = host(out)
    assert (np.abs(got - ref) <= _bound(mag, ref, K, dtype))[live].all()
    assert (got[~live] == 7.0).all()
    again = laep.moe_mx4_grouped_product(*args, out=torch.full_like(out, 7.0), **kw)
    assert torch.equal(again, out)


FFNS = [   # the two products' tiles; T, k, E, dead, d, f
    ((64, 128), (128, 256), 1000, 2, 8, 1, 7168, 640),
    ((128, 128), (64, 128), 3200, 2, 2, 0, 320, 704),
    ((128, 256), (128, 256), 1000, 8, 20, 0, 1088, 1024),
    ((128, 256), (128, 128), 8800, 1, 4, 1, 576, 1216),
    ((256, 256), (128, 256), 16500, 2, 2, 0, 576, 1024),
    ((256, 256), (128, 128), 9000, 1, 2, 0, 640, 3584)]


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("gate_up,down,T,k,E,dead,d,f", FFNS)
def test_ffn(gate_up, down, T, k, E, dead, d, f, act):
    case(f"mx4 ffn tiles={gate_up}, {down} T={T} k={k} E={E} dead={dead} d={d} f={f} act={act}")
    assert laep.laep_mx4_ffn_tile(T * k, E, d, f, act) == gate_up
    assert laep.laep_mx4_ffn_tile(T * k, E, d, f, act, down=True) == down
    x, row_src, offsets, emap, gu, dn = _ffn_inputs(T + d + f, T, k, E, dead, d, f)
    kw = dict(row_src=_i32(row_src), k=k, act_bits=act, expert_map=_i32(emap))
    args = (dev(x, torch.bfloat16), _mx4(gu), _mx4(dn), _i32(offsets))
    y, a = laep.moe_grouped_ffn_fwd_mx4(*args, save_act=act == 16, **kw)
    _ffn_check(y, x, row_src, offsets, emap, gu, dn, k, act, a)
    again, none = laep.moe_grouped_ffn_fwd_mx4(*args, **kw)
    assert none is None and torch.equal(y, again)
    own, _ = laep.moe_grouped_ffn_fwd_mx4(dev(x[row_src // k], torch.bfloat16), *args[1:],
                                          act_bits=act, expert_map=_i32(emap))
    assert torch.equal(y, own)


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("tile,T,E,N,K", [((128, 256), 8100, 20, 2048, 576),
                                          ((256, 256), 17000, 4, 3584, 640)])
def test_rows_left_and_one_expert_with_all(tile, T, E, N, K, act):
    """The large tiles where one expert has nearly every row, another one row, others none;
    rows behind the last expert and of an expert without a slot keep what they held."""
    case(f"mx4 product: one expert, rows left, tile={tile} act={act}")
    assert laep.laep_mx4_product_tile(T, E, N, K, act) == tile
    g = np.random.default_rng(T)
    sizes = np.zeros(E, np.int64)
    sizes[1], sizes[3] = 1, 300
    sizes[2] = T - 7 - 301
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    emap = np.full(E, -1, np.int32)
    emap[1], emap[2] = 1, 0
    row_src = g.permutation(T).astype(np.int32)
    x = round_bf16(g.normal(size=(T, K)))
    qw, qx = mx4.quantize(g.normal(size=(2, N, K))), mx4.quantize(x)
    xv = mx4.dequantize(*qx) if act == 4 else x
    ref, mag = mx4.grouped_product(xv[row_src], mx4.dequantize(*qw), offsets, emap)
    out = torch.full((T, N), 7.0, dtype=torch.float32, device="cuda")
    laep.moe_mx4_grouped_product(_mx4(qx) if act == 4 else dev(x, torch.bfloat16), _mx4(qw),
                                 _i32(offsets), row_src=_i32(row_src), k=1, expert_map=_i32(emap),
                                 dtype=torch.float32, out=out)
    live = int(offsets[3])
    got = host(out)
    assert (np.abs(got - ref)[:live] <= _bound(mag, ref, K, "f32")[:live]).all()
    assert (got[live:] == 7.0).all()


def _gpu_ffn(seed, T, k, E, d, f):
    """Inputs of an FFN made on the device: x, gate/up, down, offsets, row_src."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    row_src, offsets, _ = _routing(np.random.default_rng(seed), T, k, E)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)

    return (normal(T, d), laep.moe_mx4_quantize(normal(E, 2 * f, d) * d ** -0.5),
            laep.moe_mx4_quantize(normal(E, d, f) * f ** -0.5), _i32(offsets), _i32(row_src))


BIG = [((128, 256), 2100, 4, 20, 1088, 1024), ((256, 256), 16500, 2, 2, 576, 1024)]


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("tile,T,k,E,d,f", BIG)
def test_graphs_share_a_workspace(tile, T, k, E, d, f, act):
    """Two captured calls on one workspace, replayed in turn with eager calls of other sizes
    on the same workspace between: the eager results."""
    case(f"mx4 ffn in graphs, tile={tile} act={act}")
    assert laep.laep_mx4_ffn_tile(T * k, E, d, f, act) == tile
    x, gu, dn, off, src = _gpu_ffn(1, T, k, E, d, f)
    x2, _, _, off2, src2 = _gpu_ffn(2, T, k, E, d, f)
    ws = torch.full((laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, k, E, d, f),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    kw = dict(k=k, act_bits=act)
    sets = [(x, off, src), (x2, off2, src2)]
    eager = [laep.moe_grouped_ffn_fwd_mx4(a, gu, dn, o, row_src=r, **kw)[0] for a, o, r in sets]
    ys = [torch.empty_like(eager[0]) for _ in sets]
    graphs = []
    for (a, o, r), y in zip(sets, ys):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            laep.moe_grouped_ffn_fwd_mx4(a, gu, dn, o, row_src=r, ws=ws, y_perm=y, **kw)
        graphs.append(graph)
    one = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    one[E:] = 1
    for i in range(6):
        ys[i % 2].zero_()
        graphs[i % 2].replay()
        assert torch.equal(ys[i % 2], eager[i % 2])
        laep.moe_grouped_ffn_fwd_mx4(x[:1], gu, dn, one, act_bits=act, ws=ws)
        laep.moe_mx4_grouped_product(x[:700], gu, off.clamp(max=700), ws=ws)
        torch.cuda.synchronize()


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("tile,T,k,E,d,f", BIG)
def test_calls_at_once(tile, T, k, E, d, f, act):
    """Calls on two streams, each with a workspace of its own, give what they give alone."""
    case(f"mx4 ffn on two streams, tile={tile} act={act}")
    ins = [_gpu_ffn(s, T, k, E, d, f) for s in (3, 4)]
    kw = dict(k=k, act_bits=act)

    def run(v, **more):
        return laep.moe_grouped_ffn_fwd_mx4(*v[:4], row_src=v[4], **kw, **more)[0]

    alone = [run(v) for v in ins]
    ws = [torch.empty(laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, k, E, d, f),
                      dtype=torch.uint8, device="cuda") for _ in ins]
    ys = [torch.empty_like(alone[0]) for _ in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, v, w, y in zip(streams, ins, ws, ys):
            with torch.cuda.stream(s):
                run(v, ws=w, y_perm=y)
    torch.cuda.synchronize()
    for y, want in zip(ys, alone):
        assert torch.equal(y, want)
