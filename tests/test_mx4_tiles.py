"""Which tiles the products at MX4 weights take (laep_mx4_product_tile, laep_mx4_ffn_tile):
the sizes at which each was measured the fastest, and where the large ones are not possible."""
import pytest

from paper_2601_14327_amd import laep_mx4_ffn_tile as ffn_tile
from paper_2601_14327_amd import laep_mx4_product_tile as product_tile


@pytest.mark.parametrize("R,E,d,f,mx4,bf16", [
    (128, 64, 2048, 1024, (32, 64), (32, 64)),          # us 33 (64 rows: 38), bf16 37 (50)
    (1024, 64, 2048, 1024, (64, 128), (64, 128)),       # 46 (32 rows: 63), 61 (65)
    (4096, 64, 2048, 1024, (128, 256), (64, 128)),      # 60 (64: 66), 102 (BIG 128: 118)
    (12288, 64, 2048, 1024, (128, 256), (128, 256)),    # 87, 198
    (32768, 64, 2048, 1024, (128, 256), (128, 256)),
    (131072, 64, 2048, 1024, (256, 256), (256, 256)),
    (32, 16, 4096, 2048, (32, 64), (32, 64)),           # 30 (64: 36), 36 (52)
    (256, 16, 4096, 2048, (64, 128), (64, 128)),        # 42 (32: 77), 56 (75)
    (4096, 16, 4096, 2048, (128, 256), (128, 256)),     # 94 (128 x 128: 105), 222 (253)
    (131072, 4, 512, 1024, (128, 128), (128, 128)),     # k-loops too short for the large tiles
    (100, 4, 60, 64, (0, 0), (0, 0)), (-1, 4, 64, 64, (0, 0), (0, 0)),    # refused
    (1, 257, 64, 64, (0, 0), (0, 0)), (1 << 31, 4, 64, 64, (0, 0), (0, 0)),
])
def test_ffn(R, E, d, f, mx4, bf16):
    assert ffn_tile(R, E, d, f, 4) == mx4 and ffn_tile(R, E, d, f, 16) == bf16
    assert ffn_tile(R, E, d, f, 8) == (0, 0)


@pytest.mark.parametrize("N,K", [(64, 64), (192, 320), (2048, 1024), (4096, 576)])
@pytest.mark.parametrize("E", [1, 16, 256])
@pytest.mark.parametrize("act", [4, 16])
def test_more_rows_never_take_shorter_tiles(E, N, K, act):
    tiles = [product_tile(int(1.2 ** i), E, N, K, act) for i in range(80)]
    assert [t[0] for t in tiles] == sorted(t[0] for t in tiles) and tiles[0] == (32, 64)
    assert set(tiles) <= {(32, 64), (64, 128), (128, 128), (128, 256), (256, 256)}
    assert K >= 576 or tiles[-1] == (128, 128)


@pytest.mark.parametrize("R,E,N,K", [
    (1 << 28, 4, 64, 2048),             # scales of 2 GiB
    (1 << 20, 4, (1 << 20) + 64, 576),  # 32-bit offsets within a tile
])
def test_large_offsets_keep_to_the_small_tiles(R, E, N, K):
    for act in (4, 16):
        assert product_tile(R, E, N, K, act) == (128, 128)
