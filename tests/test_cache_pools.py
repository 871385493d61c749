"""Page tables of pools whose marks take most of a workgroup's LDS, and of those that are the first to take none."""
import numpy as np
import pytest

from test_cache_pages import compact, fork, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [11000, 12001, 14000, 16383, 16384, 16385, 20000])
def test_fork_and_compact(pages):
    r = np.random.default_rng(pages)
    lens = r.integers(1, 200, 300)
    table = rows(lens, 14, pages, seed=pages)
    parent = r.integers(-1, 300, 400)
    fork(table, lens, parent, np.full(400, 1000), r.integers(0, 220, 400), pages, layers=1, heads=1)
    compact(r.permutation(pages)[:pages // 3 * 2].astype(np.int32).reshape(2, -1), pages, layers=1, heads=1)
