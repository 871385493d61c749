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


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("new", [1, 40, 300])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 50)])
@pytest.mark.parametrize("what", ["queries", "keys", "both", "values", "all"])
def test_zeros(what, causal, window, new, cache):
    """Zero queries, and zero keys and values (codes of any kind with scales of zero in 8 bits), weigh all visible tokens alike."""
    p = Problem([new, 3], [77, 20], 4, 2, 128, 32, cache, seed=42)
    if what in ("queries", "both", "all"):
        p.q.zero_()
    for name in {"keys": "k", "both": "k", "values": "v", "all": "kv"}.get(what, ""):
        x = getattr(p, name + ("_scale" if cache == "s8" else ""))
        setattr(p, name + ("_scale" if cache == "s8" else ""), torch.where(x.isnan(), x, torch.zeros_like(x)))
    check(p, causal=causal, window=window)
    check(p, causal=causal, window=window, out="u8", out_scale=0.02, zero=128)


@pytest.mark.parametrize("new", [1, 40, 300])
def test_zero_columns_before_their_sequence_give_zeros(new):
    """What append makes of columns without a token (zero queries), over zero keys."""
    p = Problem([new, 5], [0, 3], 2, 1, 64, 16, "s8", seed=43)
    p.q.zero_()
    p.lens = [max(0, new - 7), 2]
    p.k_scale = torch.where(p.k_scale.isnan(), p.k_scale, torch.zeros_like(p.k_scale))
    check(p)
    check(p, causal=False)


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("new", [1, 40, 300])
@pytest.mark.parametrize("scale", [1e-9, 1e-30, 1e-45])
def test_small_scales(scale, new, cache):
    """Scores too small to tell from zero: with zero queries, and with some, all visible tokens weigh the same."""
    for zero in (True, False):
        p = Problem([new, 3], [77, 20], 4, 2, 64, 32, cache, seed=44)
        if zero:
            p.q.zero_()
        p.q[::2] *= 1e-30
        got = attend(p, scale=scale).double().numpy()
        ref, mag = p.attention(scale)
        assert (np.abs(got - ref) <= (2.0 ** -8 + 1e-4) * mag).all()
