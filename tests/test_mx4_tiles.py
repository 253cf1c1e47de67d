"""Which tiles the products at MX4 weights take (laep_mx4_product_tile, laep_mx4_ffn_tile):
the sizes at which each was measured the fastest, and where the large ones are not possible."""
import pytest

from paper_2601_14327_amd import laep_mx4_ffn_tile as ffn_tile
from paper_2601_14327_amd import laep_mx4_product_tile as product_tile


@pytest.mark.parametrize("R,E,N,K,mx4,bf16", [
    (1024, 64, 2048, 2048, (64, 128), (64, 128)),        # us 27 (128 rows: 32), 39 (59)
    (4096, 64, 2048, 2048, (64, 128), (64, 128)),        # 32 (BIG 128: 37), 59 (58)
    (8192, 64, 2048, 2048, (128, 256), (128, 256)),      # 39 (BIG 256: 53), 76 (122)
    (16384, 64, 2048, 2048, (128, 256), (128, 256)),     # 59 (BIG 256: 56), 137 (140)
    (32768, 64, 2048, 2048, (256, 256), (256, 256)),     # 89, 241 (BIG 128: 244)
    (512, 16, 4096, 4096, (128, 128), (64, 128)),        # 26 (64: 32), 53 (128: 54)
    (8192, 8, 7168, 1024, (256, 256), (256, 256)),       # 47 (BIG 128: 51), 105 (113)
    (2048, 8, 1024, 3584, (64, 128), (64, 128)),         # 15 (BIG 128: 22), 30 (44)
    (131072, 4, 1024, 512, (128, 128), (128, 128)),      # k-loops too short for the large
    (100, 4, 60, 64, (0, 0), (0, 0)), (-1, 4, 64, 64, (0, 0), (0, 0)),    # refused
    (1, 257, 64, 64, (0, 0), (0, 0)), (1 << 31, 4, 64, 64, (0, 0), (0, 0)),
])
def test_product(R, E, N, K, mx4, bf16):
    assert product_tile(R, E, N, K, 4) == mx4 and product_tile(R, E, N, K, 16) == bf16
    assert product_tile(R, E, N, K, 8) == (0, 0)


@pytest.mark.parametrize("R,E,d,f", [(128, 64, 2048, 1024), (1024, 64, 2048, 1024),
                                     (32, 16, 4096, 2048), (4096, 16, 4096, 2048),
                                     (16384, 8, 1024, 3584), (100, 4, 60, 64)])
@pytest.mark.parametrize("act", [4, 16])
def test_ffn(R, E, d, f, act):
    """Few rows: both products by 32 x 64 tiles; else each as a product of its own."""
    gate_up, down = ffn_tile(R, E, d, f, act), ffn_tile(R, E, d, f, act, down=True)
    if R <= 128:
        assert gate_up == down == ((0, 0) if d == 60 else (32, 64))
    else:
        assert gate_up == product_tile(R, E, 2 * f, d, act)
        assert down == product_tile(R, E, d, f, act)


@pytest.mark.parametrize("N,K", [(64, 64), (192, 320), (2048, 1024), (4096, 576)])
@pytest.mark.parametrize("E", [1, 16, 256])
@pytest.mark.parametrize("act", [4, 16])
def test_more_rows_keep_to_the_large_tiles(E, N, K, act):
    """From 32 rows to 64 or 128, and once tiles have 256 columns, to no smaller ones."""
    tiles = [product_tile(int(1.2 ** i), E, N, K, act) for i in range(80)]
    assert tiles[0] == (32, 64)
    assert set(tiles) <= {(32, 64), (64, 128), (128, 128), (128, 256), (256, 256)}
    order = {(32, 64): 0, (64, 128): 1, (128, 128): 1, (128, 256): 2, (256, 256): 3}
    assert [order[t] for t in tiles] == sorted(order[t] for t in tiles)
    assert K >= 576 or tiles[-1] == (128, 128)


@pytest.mark.parametrize("R,E,N,K", [
    (1 << 28, 4, 64, 2048),             # scales of 2 GiB
    (1 << 20, 4, (1 << 20) + 64, 576),  # 32-bit offsets within a tile
])
def test_large_offsets_keep_to_the_small_tiles(R, E, N, K):
    for act in (4, 16):
        assert product_tile(R, E, N, K, act) == (128, 128)
