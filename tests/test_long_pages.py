"""spmm_cache_bounds, spmm_cache_score and spmm_cache_select on the device against their definitions.

Bounds of bfloat16 caches are exact; those of 8-bit ones are one binary32 product, rounded once more to bfloat16: 2^-24 and 2^-8 of
the value.  A score is a binary32 sum of 2 head_dim products of 16-bit numbers, which are exact: each of its additions is off by at most 2^-23 (whichever way
the matrix instruction rounds) of the sum of magnitudes.  Lists are exact."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import side_stream
from long_reference import POISON, Long, ints, stream

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (8, 2, 128), (6, 2, 80), (5, 1, 16), (16, 1, 48), (40, 2, 96), (3, 3, 112), (7, 1, 32)]


def bounds(p, T=None):
    cache, batch = p.on_device()
    sp.spmm_cache_bounds(cache, p.layer, batch, T or max(1, p.tokens), stream())
    torch.cuda.synchronize()
    got, want = p.db.cpu().double(), p.bounds_wanted()
    tol = 0.0 if p.kind == "bf16" else want.abs() * (2.0 ** -8 + 2.0 ** -22)
    bad = ~(((got - want).abs() <= tol) | (got.isnan() & want.isnan()) | (got == want))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_bounds(q_heads, kv_heads, dim, page, cache):
    bounds(Long([1, 0, 5, 3 * page + 1, 1], [0, 9, page - 2, page, 5 * page + 3], q_heads, kv_heads, dim, page, cache, layers=2, layer=1, seed=1))


@pytest.mark.parametrize("T", [1, 10, 100000])
def test_bounds_whatever_the_number_of_columns_is(T):
    p = Long([40, 200, 1], [100, 0, 7], 4, 2, 64, 16, seed=2)
    bounds(p, T)
    p = Long([1, 1], [70, 3], 2, 2, 64, 16, seed=3)
    p.news, p.start = list(p.lens), np.concatenate(([0], np.cumsum(p.lens))).astype(np.int32)       # all tokens new: all pages
    bounds(p, T)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_bounds_of_what_is_not_finite(cache):
    p = Long([30, 30], [3, 3], 2, 2, 64, 16, cache, seed=4)
    at = p.table[0, 0]
    if cache == "bf16":
        p.k[0, at, 0, 2, 5], p.k[0, at, 1, 0, 7], p.k[0, at, 1, 3, 9] = float("nan"), float("inf"), -float("inf")
        p.k[0, p.table[1, 0], 0] = -0.0
    else:
        p.k_scale[0, at, 0, 2], p.k_scale[0, at, 1, 0] = float("nan"), float("inf")
        p.k_scale[0, p.table[1, 0], 0, :] = 3e38
        p.k[0, p.table[1, 0], 0, 3] = 100       # (times the scale it is not finite)
        p.k_scale[0, p.table[1, 0], 1, :] = 0.0
    bounds(p)


def test_bounds_of_sequences_that_are_not_there():
    p = Long([4, 3, 5], [20, 10, 40], 2, 2, 64, 16, seed=5, width=2)      # more tokens than the table names
    p.table[1, 0] = 10 ** 6     # a page outside the pool
    p.lens = [24, 13, 60]
    bounds(p)
    p.lens = [2, 0, -7]         # fewer tokens than columns
    bounds(p)


def test_bounds_of_any_number_of_columns():
    """The number of columns only says how many workgroups are wanted: of 64 heads more than a grid holds."""
    for T in (1, 40, 1 << 20, 1 << 40):
        bounds(Long([30, 0, 5], [50, 9, 14], 64, 64, 16, 16, seed=62), T)


def score(p, causal=True, window=0, pad=0):
    cache, batch = p.on_device()
    T, H, lds = max(1, p.tokens), p.k.shape[2], p.width + pad
    out = torch.full((T, H, lds), float(POISON), device="cuda")
    how = sp.make_select(p.q_heads, 1, 0, 0, causal, window)
    sp.spmm_cache_score(cache, p.layer, batch, p.q.cuda(), T, how, out, lds, stream())
    torch.cuda.synchronize()
    got = out.cpu().double().numpy()
    assert (got[:, :, p.width:] == POISON).all()
    got = got[:, :, :p.width]
    want, mag, mine = p.scores_wanted(causal, window)
    assert (got[~mine] == POISON).all()
    with np.errstate(invalid="ignore"):
        ok = (got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= 2 * p.dim * 2.0 ** -23 * mag)
    bad = ~ok & mine[:, None, None]
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS)
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 40)])
def test_scores(q_heads, kv_heads, dim, causal, window):
    score(Long([1] * 6, [0, 1, 31, 32, 200, 1000], q_heads, kv_heads, dim, 16, seed=6), causal, window)
    score(Long([3, 0, 70, 17, 1], [0, 5, 31, 130, 64], q_heads, kv_heads, dim, 32, layers=2, layer=1, lead=2, seed=7), causal, window, pad=3)


@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS + [(4, 2, 64), (6, 3, 128)])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 200)])
def test_scores_of_many_columns(q_heads, kv_heads, dim, causal, window):
    score(Long([300, 20, 0, 130], [700, 0, 5, 64], q_heads, kv_heads, dim, 16, lead=3, seed=61), causal, window, pad=2)


def test_scores_of_two_heads_each():
    score(Long([1] * 6, [0, 1, 31, 32, 200, 1000], 4, 2, 64, 16, seed=63))
    score(Long([3, 0, 9, 7, 1], [0, 5, 31, 130, 64], 6, 3, 112, 32, seed=64))


def test_scores_of_many_pages_and_columns():
    score(Long([1, 2], [9000, 3000], 2, 2, 64, 16, seed=8))
    score(Long([150], [2500], 2, 1, 128, 16, seed=9))


def test_scores_of_what_is_not_finite():
    p = Long([4, 1, 40], [30, 90, 64], 4, 2, 64, 16, seed=10)
    p.bounds[0, p.table[0, 0], 1, :, 3] = float("nan")
    p.q[1, 2, 5], p.q[2, 0, 6] = float("inf"), float("nan")
    p.q[3] = 0.0
    p.q[4, :, ::2] = -0.0
    score(p)


@pytest.mark.parametrize("causal", [True, False])
def test_scores_of_rows_that_see_nothing(causal):
    p = Long([4, 1, 40], [20, 0, 0], 2, 1, 64, 16, seed=11)
    p.lens = [2, 0, 7]
    score(p, causal)
    score(Long([3], [60], 2, 1, 64, 16, seed=12, width=2), causal)
    score(p, causal, (1 << 31) - 1)


def select(p, pages, first, last, causal=True, window=0, pad=0, change=None):
    cache, batch = p.on_device()
    T, H, lds = max(1, p.tokens), p.k.shape[2], p.width + pad
    scores = torch.from_numpy(p.rng.standard_normal((T, H, lds), np.float32))
    if change:
        change(scores)
    lists = torch.full((T, H, pages), POISON, dtype=torch.int32, device="cuda")
    how = sp.make_select(p.q_heads, pages, first, last, causal, window)
    sp.spmm_cache_select(cache, batch, scores.cuda(), T, lds, how, lists, stream())
    torch.cuda.synchronize()
    got, want = lists.cpu().numpy(), p.lists_wanted(scores.numpy(), pages, first, last, causal, window)
    assert (got == want).all(), (np.argwhere(got != want)[:4], got[got != want][:4], want[got != want][:4])


def small(past, news=None, page=16, seed=13, **kw):
    """A problem of long tables and hardly any memory: the rows' pages are few and repeat."""
    p = Long(news or [1] * len(past), [1] * len(past), 2, 2, 16, page, seed=seed, width=max(n // page + 2 for n in past), **kw)
    p.lens = [n + k for n, k in zip(p.news, past)]
    return p


@pytest.mark.parametrize("pages, first, last", [(1, 0, 0), (1, 0, 1), (7, 1, 2), (64, 4, 4), (100, 0, 0), (5, 3, 2)])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 900)])
def test_select(pages, first, last, causal, window):
    select(small([0, 15, 16, 100, 1000, 2047]), pages, first, last, causal, window, pad=1)
    select(small([100, 0, 900], [20, 0, 33], lead=3), pages, first, last, causal, window)


@pytest.mark.parametrize("pages_held", [129, 257, 513, 1025, 4097, 9000, 20000, 32769, 40000])
def test_select_from_long_rows(pages_held):
    select(small([16 * pages_held - 1, 16 * (pages_held // 2)]), 50, 1, 2)
    select(small([16 * pages_held - 1, 5]), pages_held - 7, 1, 2)


@pytest.mark.parametrize("pages_held", [100, 700, 3000, 6000, 10000, 20000, 40000])
def test_equal_scores_take_the_lower_page(pages_held):
    p = small([16 * pages_held])
    select(p, 33, 1, 1, change=lambda s: s.copy_((s * 2).round()))
    select(p, 33, 1, 1, change=lambda s: s.zero_())
    select(p, 33, 0, 0, change=lambda s: s.fill_(-float("inf")))
    select(p, 33, 0, 0, change=lambda s: s.copy_(torch.where(s > 0, 0.0, -0.0)))

    def odd(s):
        s[:, :, 5::9], s[:, :, 7::31], s[:, :, 8::31], s[:, :, 2::3] = float("nan"), float("inf"), -float("inf"), 1e-44 * torch.arange(s[:, :, 2::3].shape[2])
    select(p, 33, 1, 1, change=odd)
    select(p, 3, 0, 0, change=odd)


def test_select_where_nothing_is_visible():
    p = small([0, 0, 0], [4, 1, 40])
    p.lens = [2, 0, 7]
    select(p, 5, 1, 1)
    select(p, 5, 1, 1, window=(1 << 31) - 1)


def test_pages_on_another_stream_in_a_graph():
    """Bounds, scores and lists captured, and replayed with other inputs: each replay is what eager calls give."""
    p = Long([1, 3, 1], [300, 77, 1000], 8, 2, 64, 16, seed=14)
    cache, batch = p.on_device()
    T, H, how = p.tokens, 2, sp.make_select(8, 9, 1, 2)
    q, scores, lists = p.q.cuda(), torch.empty((p.tokens, 2, p.width), device="cuda"), torch.empty((p.tokens, 2, 9), dtype=torch.int32, device="cuda")

    def calls():
        sp.spmm_cache_bounds(cache, 0, batch, T, stream())
        sp.spmm_cache_score(cache, 0, batch, q, T, how, scores, p.width, stream())
        sp.spmm_cache_select(cache, batch, scores, T, p.width, how, lists, stream())

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side_stream()):
        calls()
    for i in range(3):
        q.normal_()
        p.dk.copy_(p.k.cuda() * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = p.db.clone(), scores.clone(), lists.clone()
        calls()
        torch.cuda.synchronize()
        assert torch.equal(torch.nan_to_num(got[0].float(), 5.0), torch.nan_to_num(p.db.float(), 5.0)) and torch.equal(got[1], scores) and torch.equal(got[2], lists)
    assert H == p.k.shape[2]
