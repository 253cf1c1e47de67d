"""Limits of the calls at microscaled 4-bit weights, and what looks them up (host code)."""
import pytest
import torch

import paper_2601_14327_amd as laep
from test_abi import L, _err, _fake  # noqa: F401  (L: the library fixture)


@pytest.mark.parametrize("R,f", [(1 << 28, 256), ((1 << 28) - 1, 320), (1 << 25, 2048)])
def test_no_tiles_where_the_ffn_refuses_the_rows(L, R, f):
    """H's scales in MX4, 8 bytes a row and 256 columns, are under 2 GiB."""
    E, d = 4, 64
    few = ((1 << 28) - 1) // -(-f // 256)           # the most rows that are not refused
    assert few < R
    for down in (False, True):
        assert laep.laep_mx4_ffn_tile(R, E, d, f, 4, down=down) == (0, 0)
        assert laep.laep_mx4_ffn_tile(few, E, d, f, 4, down=down) != (0, 0)
        assert laep.laep_mx4_ffn_tile(R, E, d, f, 16, down=down) != (0, 0)

    def call(R, bits):   # refused before any pointer is looked at
        return L.moe_grouped_ffn_fwd_mx4(None, 4096, 1 << 23, 64, None, None, None, None, None,
                                         None, bits, E, d, f, R, None, None, None, 0, None)
    assert call(R, 4) == 2 and "too many" in _err(L)
    assert call(few, 4) == 1 and call(R, 16) == 1      # (no offsets)


@pytest.fixture()
def ptrs():
    keep, p = _fake(65536)   # 4 MB
    yield [p + 262144 * i for i in range(15)]
    del keep


def _alias_checks(f, L, outs, ins, with_map):
    """No output or workspace over an input's first or last bytes."""
    for o in outs:
        for name, (p, n) in ins.items():
            kw = dict(em=ins["em"][0]) if with_map or name == "em" else {}
            for at in (p, p + max(n - 16, 0) // 16 * 16):
                assert f(**{o: at}, **kw) == 1 and "overlap" in _err(L), (o, name, at - p)


def test_product_buffers_that_overlap_are_refused(L, ptrs):
    x, xs, src, w, wsc, off, em, out, ws = ptrs[:9]
    T, k, E, N, K, R = 4, 2, 8, 64, 128, 8
    need = L.moe_workspace_bytes(7, T, k, E, K, N)

    def f(x=x, xs=xs, src=src, w=w, wsc=wsc, off=off, em=None, out=out, ws=ws):
        return L.moe_mx4_grouped_product(x, xs, src, T, k, w, wsc, off, em, 1, E, N, K, R, out, ws,
                                         need, None)

    # without a map the weights are all E slots, with one the first is looked at
    for slots in (E, 1):
        _alias_checks(f, L, ("out", "ws"),
                      dict(x=(x, T * K // 2), xs=(xs, T * 8), src=(src, 4 * R), off=(off, 4 * E + 4),
                           em=(em, 4 * E), w=(w, slots * N * K // 2), wsc=(wsc, slots * N * 8)),
                      slots == 1)
    assert f(out=ws) == 1 and f(ws=out) == 1 and "overlap" in _err(L)
    assert f(xs=None, out=x + 2 * T * K - 16) == 1 and f(xs=None, ws=x + 2 * T * K - 16) == 1


def test_ffn_buffers_that_overlap_are_refused(L, ptrs):
    x, src, wg, wgs, wd, wds, off, em, y, act, ws = ptrs[:11]
    T, k, E, d, ff, R = 4, 2, 8, 128, 64, 8
    need = L.moe_workspace_bytes(8, T, k, E, d, ff)

    def f(em=None, y=y, act=act, ws=ws):
        return L.moe_grouped_ffn_fwd_mx4(x, src, T, k, wg, wgs, wd, wds, off, em, 16, E, d, ff, R,
                                         y, act, ws, need, None)

    for slots in (E, 1):
        _alias_checks(f, L, ("y", "act", "ws"),
                      dict(x=(x, 2 * T * d), src=(src, 4 * R), off=(off, 4 * E + 4), em=(em, 4 * E),
                           wg=(wg, slots * ff * d), wgs=(wgs, slots * 2 * ff * 8),
                           wd=(wd, slots * ff * d // 2), wds=(wds, slots * d * 8)), slots == 1)
    assert f(act=y) == 1 and f(y=ws) == 1 and f(act=ws + need - 16) == 1 and "overlap" in _err(L)


class _Huge:
    """What the binding asks of a device tensor before it looks at its memory."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, *shape, dtype=torch.uint8):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 64])
def test_sizes_past_a_c_int_are_refused(n):
    """(The C calls would be passed their low 32 bits: 64 columns of 2^32 + 64.)"""
    bf16, off = torch.bfloat16, torch.zeros(2, dtype=torch.int32)

    def w(N, K):
        return laep.Mx4(_Huge(1, N, K // 2), _Huge(1, -(-K // 256), N, 8))

    def x(T, K):
        return _Huge(T, K, dtype=bf16)

    for call in (lambda: laep.moe_mx4_quantize(x(1, n)),
                 lambda: laep.moe_mx4_quantize(_Huge(n, 1, 32, dtype=bf16)),
                 lambda: laep.moe_mx4_dequantize(_Huge(1, n // 2), _Huge(n // 256 + 1, 1, 8)),
                 lambda: laep.moe_mx4_dequantize(_Huge(n, 1, 16), _Huge(n, 1, 1, 8)),
                 lambda: laep.moe_mx4_grouped_product(x(n, 64), w(64, 64), off),
                 lambda: laep.moe_mx4_grouped_product(x(8, n), w(64, n), off),
                 lambda: laep.moe_mx4_grouped_product(x(8, 64), w(n, 64), off),
                 lambda: laep.moe_mx4_grouped_product(x(8, 64), w(64, 64), off, k=n),
                 lambda: laep.moe_grouped_ffn_fwd_mx4(x(n, 64), w(128, 64), w(64, 64), off),
                 lambda: laep.moe_grouped_ffn_fwd_mx4(x(8, n), w(128, n), w(n, 64), off),
                 lambda: laep.moe_grouped_ffn_fwd_mx4(x(8, 64), w(2 * n, 64), w(64, n), off),
                 lambda: laep.moe_grouped_ffn_fwd_mx4(x(8, 64), w(128, 64), w(64, 64), off, k=n)):
        with pytest.raises(ValueError, match=f"={n} is past"):
            call()
