"""spmm_cache_attend_selected on the device where nothing is rounded to less than binary32: tolerances as derived in long_exact.py."""
import numpy as np
import pytest

from long_exact import MANY, ODD, compare, limits, plant
from long_reference import POISON, Long
from test_long_attend import attend, random_lists
from test_long_emulated import FORMS

gpu = pytest.mark.gpu


def held(p, lists, scale, causal=True, window=0):
    got = attend(p, lists, scale=scale, causal=causal, window=window).double().numpy()
    ref, tol = limits(p, lists, scale, causal, window)
    none = np.isnan(ref)
    assert (got[none] == POISON).all()
    bad = ~none & ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3], tol[bad][:3])


@gpu
@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("news, q_heads, kv_heads, dim", FORMS)
def test_weights_of_values_are_not_rounded(news, q_heads, kv_heads, dim, cache):
    """Few tokens with small scores, whose weights are all alike."""
    p = Long(news, [20] * len(news), q_heads, kv_heads, dim, 16, cache, seed=4)
    held(p, random_lists(p, 2), 0.01)


@gpu
@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("news, past, page, pages, causal, window", [([1, 1], 900, 64, 9, True, 0), ([3], 3000, 16, 150, False, 0), ([70], 400, 32, 7, True, 90), ([300], 500, 64, 3, True, 0)])
def test_longer_lists_and_larger_scores(news, past, page, pages, causal, window, cache):
    p = Long(news, [past] * len(news), 8, 4, 64, page, cache, seed=5)
    lists = random_lists(p, pages, causal, window)
    for scale in (0.02, 0.125):
        held(p, lists, scale, causal, window)


@gpu
@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("q_heads, kv_heads, dim, new", MANY)
@pytest.mark.parametrize("causal, window, pages", [(True, 0, 4), (True, 33, 9), (False, 0, 20)])
def test_odd_scales_in_lists_of_8_bit_caches(q_heads, kv_heads, dim, new, causal, window, pages, odd):
    """Lists that have a wave or four each, in which columns share a softmax over streams of keys."""
    p = Long([new], [60], q_heads, kv_heads, dim, 16, "s8", seed=6)
    plant(p, odd)
    lists = random_lists(p, pages, causal, window)
    bad = compare(attend(p, lists, scale=0.02, causal=causal, window=window).double().numpy(), p, lists, 0.02, causal, window)
    assert bad[0] == 0, bad
