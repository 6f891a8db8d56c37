"""CPU: the rule that cuts an 8-bit product (csrc/matmul_i8_plan.h), and that the products of the GPU tests reach all it can choose."""
import pytest

from matmul_plans import PRODUCTS, TILES, plan


@pytest.mark.parametrize("m,n,k,tile,splits", PRODUCTS)
def test_plans_of_the_products_of_the_tests(m, n, k, tile, splits):
    assert plan(m, n, k) == (tile, splits)


def test_the_products_of_the_tests_take_every_tile_whole_and_split():
    taken = {(tile, splits > 1) for *_, tile, splits in PRODUCTS}
    assert taken == {(t, False) for t in TILES} | {(t, True) for t in ("64x64", "64x128", "128x128")}
    assert {splits for *_, splits in PRODUCTS} == set(range(1, 9))
    for tile, (bm, bn) in TILES.items():        # and each with a last row tile and a last column tile that are not full
        of = [p for p in PRODUCTS if p[3] == tile]
        assert any(m % bm and n % bn for m, n, *_ in of), tile


@pytest.mark.parametrize("k", [1, 128, 257, 384, 385, 1000, 4096, 130944])
def test_a_split_is_never_shorter_than_the_ring_and_fits_the_workspace(k):
    kt = -(-k // 128)
    for m in (1, 17, 64, 65, 127, 128, 129, 300, 600, 1000, 2000, 4096, 100000):
        for n in (1, 15, 64, 65, 128, 1000, 2053, 4096, 14336, 100000):
            tile, splits = plan(m, n, k)
            assert (tile == "short") == (kt < 3)
            assert 1 <= splits <= 8 and (splits == 1 or kt // splits >= 3)
            assert splits == 1 or splits * m * (-(-n // 4) * 4) * 4 <= 64 << 20
