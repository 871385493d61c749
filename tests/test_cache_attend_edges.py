"""spmm_cache_attend on the device where its numbers lie at an edge: windows as wide as an int, zero queries and scales, and values
that are not finite in either type of cache.  Tolerances are those of test_cache_attend.py."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import Problem
from test_cache_attend import attend, check

pytestmark = pytest.mark.gpu

CACHES = ["bf16", "s8"]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("new", [9, 60])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_as_wide_as_an_int(new, causal, cache):
    """Also where the first columns lie before their sequence."""
    p = Problem([new, new], [40, 0], 2, 1, 64, 16, cache, seed=41)
    p.lens = [new + 40, new - 5]
    check(p, causal=causal, window=(1 << 31) - 1)
    check(p, causal=causal, window=(1 << 31) - 7)
