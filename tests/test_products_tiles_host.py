"""The sizes that the tests of every tile use are of the tiles that they are for."""
from test_gpu_products_paths import DW, DW_CASES, DX, DX_CASES, GATED, GATED_CASES, I8, I8_CASES, I8_GATED, I8_GATED_CASES, PAIRS, _pair, tile_of


def test_the_cases_take_the_tiles_they_are_for():
    for kind, cases in ((I8, I8_CASES), (I8_GATED, I8_GATED_CASES), (GATED, GATED_CASES), (DX, DX_CASES), (DW, DW_CASES)):
        for tile, splits, *size in cases:
            assert tile_of(kind, *size) == (tile, splits), (kind, size)
            if kind in (DX, DW):
                assert _pair(*size) < 0, size
    for tile, *size in PAIRS:
        assert _pair(*size) == tile, size
