"""Refusals of the calls at microscaled 4-bit weights (laep_mx4.h), on the host: an
invalid call returns its code before any HIP call; and what the binding refuses."""
import pytest
import torch

import paper_2601_14327_amd as laep
from paper_2601_14327_amd import api
from test_abi import L, _err, _fake  # noqa: F401  (L: the library fixture)


@pytest.fixture()
def ptrs():
    keep, p = _fake(4096)   # 256 KB
    yield [p + 16384 * i for i in range(16)]
    del keep


def test_quantize_refusals(L, ptrs):
    s, c, e = ptrs[:3]

    def quant(src=s, dt=1, n=1, R=4, C=64, codes=c, scale=e):
        return L.moe_mx4_quantize(src, dt, n, R, C, codes, scale, None)

    def back(codes=c, scale=e, dt=1, n=1, R=4, C=64, out=s):
        return L.moe_mx4_dequantize(codes, scale, dt, n, R, C, out, None)

    for f in (quant, back):
        assert f(dt=2) == 2 and "dtype" in _err(L)
        assert f(C=48) == 1 and "multiple of 32" in _err(L)
        assert f(C=0) == 1 and f(R=-1) == 1 and f(R=1 << 31) == 1 and f(n=-1) == 1
        assert f(codes=None) == 1 and f(scale=None) == 1 and "non-null" in _err(L)
        assert f(codes=c + 4) == 1 and f(scale=e + 8) == 1 and "aligned" in _err(L)
        assert f(R=0) == 0 and f(n=0) == 0        # nothing to do: nothing is enqueued
    assert quant(src=None) == 1 and quant(src=s + 2) == 1
    assert quant(codes=s) == 1 and "overlap" in _err(L)
    assert quant(scale=s + 496) == 1 and quant(codes=s + 496) == 1
    assert quant(scale=c + 112) == 1
    assert back(out=None) == 1 and back(out=s + 8) == 1
    assert back(out=c) == 1 and "overlap" in _err(L) and back(scale=s + 496) == 1


def test_product_refusals(L, ptrs):
    x, xs, src, w, wsc, off, out, ws = ptrs[:8]

    def f(x=x, xs=xs, src=src, T=4, k=2, w=w, wsc=wsc, off=off, em=None, dt=1, E=8, N=64, K=128,
          R=8, out=out, ws=ws, n=1 << 20):
        return L.moe_mx4_grouped_product(x, xs, src, T, k, w, wsc, off, em, dt, E, N, K, R, out,
                                         ws, n, None)

    assert f(dt=3) == 2 and f(E=0) == 1 and f(E=257) == 1 and "E=257" in _err(L)
    assert f(N=96) == 2 and f(K=32) == 2 and "multiples of 64" in _err(L)
    assert f(N=0) == 1 and f(K=-64) == 1
    assert f(T=-1) == 1 and f(k=0) == 1
    assert f(R=9) == 1 and "T*k" in _err(L)
    assert f(src=None, R=5) == 1 and "without row_src" in _err(L)
    assert f(R=-1) == 1 and f(T=1 << 30, k=4, R=1 << 31) == 1
    assert f(N=1 << 17, K=1 << 15) == 2 and "2 GiB" in _err(L)
    assert f(T=1 << 25, k=1) == 2 and "activations" in _err(L)          # 2^25 x 128 / 2 bytes
    assert f(T=1 << 23, xs=None, k=1) == 2
    assert f(off=None) == 1 and f(x=None) == 1 and f(w=None) == 1 and f(wsc=None) == 1
    assert f(out=None) == 1 and f(x=x + 8) == 1 and f(xs=xs + 4) == 1 and f(out=out + 2) == 1
    assert "aligned" in _err(L)
    assert f(out=x) == 1 and "overlap" in _err(L)
    assert f(out=xs) == 1 and f(out=w) == 1 and f(out=wsc) == 1
    assert f(xs=None, out=x + 1008) == 1
    assert f(R=0, x=None, w=None, wsc=None, out=None, ws=None, n=0) == 0
    need = L.moe_workspace_bytes(7, 4, 2, 8, 128, 64)
    if need:
        assert f(n=need - 1) == 3 and "workspace" in _err(L) and f(ws=None) == 1


def test_ffn_refusals(L, ptrs):
    x, src, wg, wgs, wd, wds, off, y, act, ws = ptrs[:10]
    need = L.moe_workspace_bytes(8, 4, 2, 8, 128, 64)
    assert 0 < need <= 16384

    def f(x=x, src=src, T=4, k=2, wg=wg, wgs=wgs, wd=wd, wds=wds, off=off, em=None, bits=16, E=8,
          d=128, f=64, R=8, y=y, act=None, ws=ws, n=need):
        return L.moe_grouped_ffn_fwd_mx4(x, src, T, k, wg, wgs, wd, wds, off, em, bits, E, d, f, R,
                                         y, act, ws, n, None)

    assert f(bits=8) == 2 and "act_bits=8" in _err(L)
    assert f(bits=4, act=act) == 2 and "act_save" in _err(L)
    assert f(E=300) == 1 and f(d=96) == 2 and f(f=32) == 2 and f(d=0) == 1
    assert f(T=-1) == 1 and f(k=0) == 1 and f(R=9) == 1 and f(src=None, R=5) == 1
    assert f(d=1 << 15, f=1 << 16) == 2 and f(T=1 << 24, k=1) == 2 and "2 GiB" in _err(L)
    assert f(T=1 << 22, k=64, R=1 << 28, bits=4) == 2 and "too many" in _err(L)
    for name in ("x", "wg", "wgs", "wd", "wds", "off", "y", "ws"):
        assert f(**{name: None}) == 1, name
    for name, p in (("x", x), ("wg", wg), ("wgs", wgs), ("wd", wd), ("wds", wds), ("y", y),
                    ("ws", ws), ("act", act)):
        assert f(**{name: p + 8}) == 1 and "aligned" in _err(L), name
    assert f(n=need - 1) == 3 and "workspace" in _err(L)
    for p in (x, wg, wgs, wd, wds, ws):
        assert f(y=p) == 1 and "overlap" in _err(L)
        assert f(act=p) == 1 and "overlap" in _err(L)
    assert f(act=y) == 1 and "act_save" in _err(L)
    assert f(R=0, x=None, y=None, ws=None, n=0) == 0


def test_workspaces_grow_with_the_tokens():
    n = [laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, 2, 8, 320, 192) for T in range(300)]
    assert all(a <= b for a, b in zip(n, n[1:]))
    n = [laep.workspace_bytes(laep.LAEP_CALL_MX4_PRODUCT, T, 2, 8, 320, 192) for T in range(300)]
    assert all(a <= b for a, b in zip(n, n[1:]))
    assert laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, -1, 2, 8, 320, 192) == 0


def test_host_tensors_and_other_layouts_are_refused():
    u8, bf = torch.uint8, torch.bfloat16
    x = torch.zeros(4, 64, dtype=bf)
    with pytest.raises(ValueError, match="src must be a device tensor"):
        laep.moe_mx4_quantize(x)
    with pytest.raises(ValueError, match="codes must be a device tensor"):
        laep.moe_mx4_dequantize(torch.zeros(4, 32, dtype=u8), torch.zeros(1, 4, 8, dtype=u8))
    w = laep.Mx4(torch.zeros(1, 64, 32, dtype=u8), torch.zeros(1, 1, 64, 8, dtype=u8))
    off = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        laep.moe_mx4_grouped_product(x, w, off)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        laep.moe_grouped_ffn_fwd_mx4(x, w, w, off)
    with pytest.raises(ValueError, match="must be an Mx4"):
        api._need_mx4(torch.zeros(1, 64, 32, dtype=u8), "w", (1,), 64, 64, x.device)
    with pytest.raises(ValueError, match=r"w.codes must be torch.uint8 \(1, 64, 64\)"):
        api._need_mx4(w, "w", (1,), 64, 128, x.device)


@pytest.mark.gpu
def test_device_tensors_of_other_kinds_are_refused():
    def z(*s, dt=torch.uint8):
        return torch.zeros(s, dtype=dt, device="cuda")

    bf, i32 = torch.bfloat16, torch.int32
    with pytest.raises(laep.LaepError, match="dtype"):
        laep.moe_mx4_quantize(z(4, 64, dt=torch.float16))
    with pytest.raises(laep.LaepError, match="multiple of 32"):
        laep.moe_mx4_quantize(z(4, 48, dt=bf))
    with pytest.raises(ValueError, match="contiguous"):
        laep.moe_mx4_quantize(z(4, 128, dt=bf)[:, :64])
    with pytest.raises(ValueError, match="rows and columns"):
        laep.moe_mx4_quantize(z(64, dt=bf))
    with pytest.raises(ValueError, match="scale"):
        laep.moe_mx4_quantize(z(4, 64, dt=bf), scale=z(4, 2))
    with pytest.raises(ValueError, match="scale"):
        laep.moe_mx4_dequantize(z(4, 32), z(4, 1, 8))
    w = laep.Mx4(z(2, 64, 64), z(2, 1, 64, 8))
    x, off, src = z(4, 128, dt=bf), z(3, dt=i32), z(8, dt=i32)
    ok = dict(row_src=src, k=2)
    for bad, match in ((dict(offsets=z(3, dt=torch.int64)), "offsets"),
                       (dict(offsets=z(4, dt=i32)), "expert_map"),
                       (dict(row_src=z(8, dt=torch.int64), k=2), "row_src"),
                       (dict(expert_map=z(3, dt=i32)), "expert_map"),
                       (dict(x=z(4, 192, dt=bf)), "w.codes"), (dict(x=z(4, 128, dt=torch.float32)), "x"),
                       (dict(w=laep.Mx4(z(2, 64, 64), z(2, 64, 8))), "w.scale"),
                       (dict(x=laep.Mx4(z(4, 64), z(4, 1, 8))), "x.scale"),
                       (dict(out=z(8, 64, dt=torch.float32)), "out"),
                       (dict(out=z(8, 128, dt=bf)[:, :64]), "out"),
                       (dict(ws=torch.zeros(1 << 20, dtype=torch.uint8)), "ws")):
        a = dict(dict(x=x, w=w, offsets=off, **ok), **bad)
        with pytest.raises(ValueError, match=match):
            laep.moe_mx4_grouped_product(a.pop("x"), a.pop("w"), a.pop("offsets"), **a)
    with pytest.raises(laep.LaepError, match="unsupported dtype"):
        laep.moe_mx4_grouped_product(x, w, off, dtype=torch.float16, **ok)
    with pytest.raises(laep.LaepError, match="T\\*k"):
        laep.moe_mx4_grouped_product(x, w, off, row_src=src, k=1)
    wg, wd = laep.Mx4(z(2, 128, 64), z(2, 1, 128, 8)), laep.Mx4(z(2, 128, 32), z(2, 1, 128, 8))
    for bad, match in ((dict(w_down=laep.Mx4(z(3, 128, 32), z(3, 1, 128, 8))), "w_gate_up"),
                       (dict(w_gate_up=laep.Mx4(z(2, 64, 64), z(2, 1, 64, 8))), "w_gate_up"),
                       (dict(w_gate_up=wg.codes), "Mx4"),
                       (dict(act_save=z(8, 64, dt=bf)), "act_save"),
                       (dict(y_perm=z(8, 64, dt=bf)), "y_perm"), (dict(x=z(4, 64, dt=bf)), "w_gate_up")):
        a = dict(dict(x=x, w_gate_up=wg, w_down=wd, offsets=off, **ok), **bad)
        with pytest.raises(ValueError, match=match):
            laep.moe_grouped_ffn_fwd_mx4(a.pop("x"), a.pop("w_gate_up"), a.pop("w_down"),
                                         a.pop("offsets"), **a)
    with pytest.raises(laep.LaepError, match="act_save"):
        laep.moe_grouped_ffn_fwd_mx4(x, wg, wd, off, act_bits=4, save_act=True, **ok)
    with pytest.raises(laep.LaepError, match="workspace"):
        laep.moe_grouped_ffn_fwd_mx4(x, wg, wd, off, ws=z(16), **ok)


def test_workspaces_grow_with_the_rows_past_32_bits():
    """More tiles than 2^31 (no buffer holds their output): the size does not wrap."""
    product = [laep.workspace_bytes(laep.LAEP_CALL_MX4_PRODUCT, T, 64, 4, 576, 1 << 20)
               for T in (1 << 18, 1 << 20, 1 << 22, 1 << 24)]
    ffn = [laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, 64, 4, 576, 1 << 19)
           for T in (1 << 18, 1 << 20, 1 << 22, 1 << 24)]
    for sizes in (product, ffn):
        assert all(3.9 < b / a < 4.1 for a, b in zip(sizes, sizes[1:]))
