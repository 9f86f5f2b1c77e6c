"""Sizes that other tests need as products in two parts are."""
import pytest

from test_block_matmul_plans import plan  # noqa: F401


@pytest.mark.parametrize("m,k,n", [(18, 4096, 19000), (36, 4096, 20001), (100, 4096, 20001), (65, 4096, 22016), (100, 4096, 19000)])
def test_rows_that_are_written_again(plan, m, k, n):  # noqa: F811
    p = plan(m, n, k)
    assert not p["pairs"] and p["parts"][1][1] > 0


def test_parts_that_go_in_one_launch(plan):  # noqa: F811
    """Clusters of the second part's size whose CTAs have a tile each of the first: every tile once, no cluster without one, and a grid that can be."""
    for m in (1, 18, 36, 48):
        for n in (19000, 22016, 37889, 56833, 65535 * 128):
            for k in (16, 128, 256, 640, 1280, 4096, 11008):
                (first, count, _), (begin, rest, size) = plan(m, n, k)["parts"]
                if rest == 0:
                    continue
                alone = -(-count // size)
                tiles = [t for t in range(alone * size) if t < begin] + [begin + y for y in range(rest)]
                assert first == 0 and tiles == list(range(-(-n // 128))) and (alone - 1) * size < begin and alone + rest <= 65535


@pytest.mark.parametrize("m,k,n", [(18, 1280, 38016), (18, 1280, 60160), (9, 4096, 76800), (36, 1280, 60160)])
def test_more_tiles_than_clusters_of_one_launch_hold(plan, m, k, n):  # noqa: F811
    """Up to 48 rows two parts are for one tile an SM: of more the clusters would not all fit at once."""
    assert plan(m, n, k)["parts"][1][1] == 0
