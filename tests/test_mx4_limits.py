"""Limits of the calls at microscaled 4-bit weights, and what looks them up (host code)."""
import pytest

import paper_2601_14327_amd as laep
from test_abi import L, _err  # noqa: F401  (L: the library fixture)


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
