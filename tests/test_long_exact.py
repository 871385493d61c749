"""spmm_cache_attend_selected on the device where nothing is rounded to less than binary32, tolerances as derived in long_exact.py, and spmm_cache_weigh where rows share
pages, with the tolerance of test_long_attend.py."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from long_exact import MANY, ODD, SHARED, compare, limits, plant, share, shared_weights
from long_reference import POISON, Long, stream
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


def weights(p, max_new, window, times=1, scale=None):
    cache, batch = p.on_device()
    how = sp.make_weigh(p.q_heads, max_new, scale or p.dim ** -0.5, True, window, 0.5)
    work = torch.full((sp.spmm_weigh_work_bytes(cache, batch, p.tokens, how),), 255, dtype=torch.uint8, device="cuda")
    q, old = p.q.cuda(), p.dw.clone()
    for _ in range(times):
        p.dw.copy_(old)
        sp.spmm_cache_weigh(cache, p.layer, batch, q, p.tokens, how, work, stream())
        torch.cuda.synchronize()
        yield p.dw.cpu().double().numpy()


@gpu
@pytest.mark.parametrize("q_heads, kv_heads, dim, page, cache", [(4, 2, 64, 16, "bf16"), (2, 2, 32, 16, "s8"), (20, 1, 80, 16, "bf16"), (8, 2, 128, 64, "s8"), (6, 3, 48, 256, "bf16"),
                                                                 (32, 8, 128, 32, "bf16"), (64, 8, 96, 16, "s8")])
@pytest.mark.parametrize("news, pasts, shared", SHARED + [([1] * 40, [300] * 40, [(0, list(range(1, 40)), 16), (7, list(range(8, 20)), 18)]), ([7] * 20, [500] * 20, [(0, list(range(1, 20)), 28)])])
def test_weights_of_shared_pages(news, pasts, shared, q_heads, kv_heads, dim, page, cache):
    """As forks leave them: every row's attention counts, the weight fades once, and the result is the same each time."""
    if page > 16:
        pasts = [past * page // 16 for past in pasts] if len(news) < 10 else pasts
        shared = shared if len(news) < 10 else [(a, b, c * 16 // page) for a, b, c in shared]
    p = Long(news, pasts, q_heads, kv_heads, dim, page, cache, layers=2, layer=1, seed=7)
    share(p, shared)
    window = page * 5 if dim == 32 else 0
    want, added = shared_weights(p, 8, dim ** -0.5, True, window, 0.5)
    first = None
    for got in weights(p, 8, window, times=3):
        bad = ~(np.abs(got - want) <= 3e-4 * added + 2.0 ** -22 * np.abs(want))
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])
        assert first is None or (got == first).all()
        first = got


@gpu
@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("news, pasts, q_heads, kv_heads, dim, page, window", [
    ([1, 1, 3], [300, 40, 700], 4, 2, 64, 16, 0), ([1], [3000], 8, 1, 128, 64, 0), ([30, 7], [50, 600], 6, 2, 80, 16, 0), ([100], [900], 32, 4, 128, 32, 250), ([5] * 9, [1500] * 9, 16, 8, 32, 64, 0)])
def test_weights_are_off_by_what_binary32_is(news, pasts, q_heads, kv_heads, dim, page, window, cache):
    p = Long(news, pasts, q_heads, kv_heads, dim, page, cache, seed=8)
    for scale in (0.01, 0.1):
        tol = np.zeros(p.weight.shape)
        want, _ = shared_weights(p, 40, scale, True, window, 0.5, tol)
        got, = weights(p, 40, window, scale=scale)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], tol[bad][:3])


@gpu
@pytest.mark.parametrize("q_heads, kv_heads, dim", [(8, 2, 64), (16, 4, 128), (40, 2, 48)])
def test_scores_of_a_mixed_batch_are_those_of_two_calls(q_heads, kv_heads, dim):
    p = Long([1] * 40 + [90], [300] * 41, q_heads, kv_heads, dim, 16, seed=10)
    cache, whole = p.on_device()
    start, lens, table = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (p.start, p.lens, p.table))
    how, q, width, T = sp.make_select(q_heads, 1, 0, 0, True, 0), p.q.cuda(), p.width, p.tokens
    one, two = (torch.zeros((T, kv_heads, width), device="cuda") for _ in range(2))
    sp.spmm_cache_score(cache, 0, whole, q, T, how, one, width, stream())
    sp.spmm_cache_score(cache, 0, sp.make_batch(start[:41], lens[:40], table[:40]), q, 40, how, two, width, stream())
    sp.spmm_cache_score(cache, 0, sp.make_batch(start[40:] - 40, lens[40:], table[40:]), q[40:], T - 40, how, two[40:], width, stream())
    torch.cuda.synchronize()
    assert torch.equal(one, two)
