"""spmm_cache_attend_selected and spmm_cache_weigh on the device against their definitions.

Attention: tolerances are those of test_cache_attend.py (weights rounded to bfloat16 once, 2^-8 of sum p |v|; results to their type).
Weights: a score is a binary32 sum of head_dim exact products and is off by at most head_dim 2^-23 sum |q k| scale; scores here stay below 40 (their
magnitudes' sums below 100), so that a power is off by a relative 128 * 2^-23 * 100 = 1.5e-3 at most, and typically, as errors are of both signs,
by a hundredth of it.  3e-4 of what a call adds to a weight, on both sides of the softmax, is held here; what it was before is one product and one sum: 2^-23."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import side_stream
from long_reference import OUT, POISON, Long, ints, stream

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (8, 2, 128), (6, 2, 80), (5, 1, 16), (16, 1, 64), (20, 1, 96), (40, 2, 32)]


def random_lists(p, pages, causal=True, window=0, seed=0):
    """For each column and head, pages that it sees in part, in order, then -1."""
    r = np.random.default_rng(seed)
    lists = np.full((max(1, p.tokens), p.k.shape[2], pages), -1, np.int32)
    for t, b, at in p.columns():
        lo, hi = p.pages_seen(b, at, causal, window)
        for h in range(lists.shape[1]):
            n = min(pages, max(0, hi - lo + 1))
            lists[t, h, :n] = np.sort(r.permutation(np.arange(lo, hi + 1))[:n])
    return lists


def attend(p, lists, out="f32", out_scale=1.0, zero=0, causal=True, window=0, pad=0, scale=None):
    cache, batch = p.on_device()
    T, pages = max(1, p.tokens), lists.shape[2]
    how = sp.make_attend(p.q_heads, max(p.news + [1]), scale or p.dim ** -0.5, causal, window, out, out_scale, zero)
    o = torch.full((p.q_heads * p.dim, T + pad), POISON, dtype=OUT[out], device="cuda")
    work = torch.full((sp.spmm_selected_work_bytes(cache, T, how, pages),), 255, dtype=torch.uint8, device="cuda")     # (NaN)
    sp.spmm_cache_attend_selected(cache, p.layer, batch, p.q.cuda(), T, how, ints(lists), pages, o, T + pad, work, stream())
    torch.cuda.synchronize()
    o = o.cpu()
    assert (o[:, T:] == POISON).all()
    return o[:, :T]


def check(p, lists, out="f32", out_scale=1.0, zero=0, scale=None, **kw):
    got = attend(p, lists, out, out_scale, zero, scale=scale, **kw).double().numpy()
    kw.pop("pad", None)
    ref, mag = p.selected_wanted(lists, scale or p.dim ** -0.5, **kw)
    mine = np.zeros(got.shape[1], bool)
    mine[[t for t, _, _ in p.columns()]] = True
    assert (got[:, ~mine] == POISON).all()
    tol = (2.0 ** -8 + 1e-4) * mag
    if out == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    if out in ("s8", "u8"):
        lo, hi = (-128, 127) if out == "s8" else (0, 255)
        edge = lambda x: np.clip(np.rint(x / out_scale) + zero, lo, hi)     # noqa: E731
        bad = mine & ~((got >= edge(ref - tol)) & (got <= edge(ref + tol)))
    else:
        with np.errstate(invalid="ignore"):
            bad = mine & ~((np.abs(got - ref) <= tol) | (got == ref) | (np.isnan(got) & np.isnan(ref)))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_one_token_each(q_heads, kv_heads, dim, page, cache):
    p = Long([1] * 7, [0, 1, 15, 16, 63, 200, 1000], q_heads, kv_heads, dim, page, cache, layers=2, layer=1, seed=1)
    for pages in (1, 5, 40):
        check(p, random_lists(p, pages))


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS[:3])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 23), (False, 40), (True, 1)])
def test_chunks_behind_a_past(q_heads, kv_heads, dim, causal, window, cache):
    p = Long([3, 0, 40, 17, 1], [0, 5, 31, 130, 64], q_heads, kv_heads, dim, 32, cache, lead=2, seed=2)
    check(p, random_lists(p, 3, causal, window), causal=causal, window=window)
    # pages in any order, without regard to what is visible, some named by no number
    lists = np.random.default_rng(3).integers(-3, p.width + 2, (p.tokens, kv_heads, 6)).astype(np.int32)
    lists[:, :, 2] = 1 << 30
    lists[:, :, 4] = -(1 << 31)
    check(p, lists, causal=causal, window=window)


@pytest.mark.parametrize("page, pages", [(16, 1), (16, 2), (16, 130), (32, 7), (128, 3), (256, 2), (256, 1), (16, 1500)])
@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_lists_of_all_lengths(page, pages, cache):
    p = Long([1, 2], [page * 9 + 3, 5], 4, 2, 64, page, cache, seed=4)
    check(p, random_lists(p, pages))
    p = Long([1], [min(page * pages * 2, 8000)], 2, 1, 128, page, cache, seed=5)
    check(p, random_lists(p, pages))


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim, new", [(4, 4, 64, 300), (8, 4, 128, 240), (20, 5, 80, 188), (40, 2, 96, 240), (12, 12, 16, 90), (16, 2, 48, 480)])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 50), (True, 23)])
def test_many_lists(q_heads, kv_heads, dim, new, causal, window, cache):
    """A thousand or so, which have a wave each in 8 bits: of two sequences, with columns of no sequence before them, and of none at a position."""
    p = Long([new, 7], [150, 0], q_heads, kv_heads, dim, 16, cache, lead=1, seed=31)
    p.lens[1] = 4
    for pages in (1, 6):
        check(p, random_lists(p, pages, causal, window, seed=pages), causal=causal, window=window)
    lists = np.random.default_rng(3).integers(-3, p.width + 2, (p.tokens, kv_heads, 9)).astype(np.int32)
    check(p, lists, out="bf16", causal=causal, window=window, pad=2)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim, new", [(4, 4, 64, 70), (8, 4, 128, 65), (20, 5, 80, 60), (40, 2, 96, 45), (12, 12, 16, 22), (16, 2, 48, 140), (32, 2, 128, 130)])
@pytest.mark.parametrize("page, pages", [(16, 40), (64, 9), (32, 1)])
def test_lists_of_a_workgroup_each(q_heads, kv_heads, dim, new, page, pages, cache):
    """A few hundred lists, shorter and longer than the steps of a workgroup's waves."""
    for causal, window in ((True, 0), (False, 50)):
        p = Long([new, 3], [600, 20], q_heads, kv_heads, dim, page, cache, seed=66)
        lists = random_lists(p, pages, causal, window, seed=67)
        lists[1], lists[2, 0, 1:] = -1, -1
        check(p, lists, causal=causal, window=window)


def test_lists_of_many_pages():
    p = Long([130], [3000], 2, 2, 32, 16, "s8", seed=68)
    check(p, random_lists(p, 1000, seed=69))


@pytest.mark.parametrize("causal", [True, False])
def test_windows_behind_what_the_table_names(causal):
    """Positions beyond the row's width, whose windows begin at its end or behind it: nothing is visible."""
    p = Long([3], [60], 2, 1, 64, 16, seed=32, width=2)
    lists = np.tile(np.arange(2, dtype=np.int32), (3, 1, 1))
    for window in (1, 28, 29, 30, 31, 32, 63):
        check(p, lists, causal=causal, window=window)


@pytest.mark.parametrize("news", [[1], [40, 3]])
@pytest.mark.parametrize("out, scale, zero", [("bf16", 1, 0), ("s8", 0.02, 3), ("u8", 0.02, 128), ("f32", 1, 0)])
def test_output_types_and_pitches(news, out, scale, zero):
    p = Long(news, [1000] * len(news), 4, 2, 64, 32, seed=6)
    check(p, random_lists(p, 20), out=out, out_scale=scale, zero=zero, pad=5)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_rows_that_see_nothing_and_lists_of_nothing(cache):
    p = Long([4, 1, 40], [20, 0, 0], 2, 1, 64, 16, cache, seed=7)
    p.lens = [2, 0, 7]        # more columns than tokens: the first ones lie before the sequence
    lists = np.tile(np.arange(4, dtype=np.int32), (p.tokens, 1, 1))
    check(p, lists)
    check(p, lists, causal=False)
    p = Long([3, 1], [600, 2000], 2, 1, 64, 16, cache, seed=8)
    lists = np.full((4, 1, 90), -1, np.int32)
    check(p, lists)
    lists[:, :, 70] = 1
    check(p, lists)
    lists[:, :, :] = 2      # one page 90 times
    check(p, lists)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("news", [[1], [20]])
def test_what_is_not_finite(news, cache):
    """In hidden places it has no influence; in visible ones it reaches the columns that see it."""
    p = Long(news, [200], 4, 1, 64, 16, cache, seed=9)
    lists = random_lists(p, 13)
    seen = p.selected_wanted(lists, 0.125)[0]
    assert np.isfinite(seen).all()
    last = p.table[0, (p.lens[0] - 1) // 16]
    first = p.table[0, 0]
    if cache == "bf16":
        p.v[0, last, 0, :, (p.lens[0] - 1) % 16] = float("inf")       # the last token: the last column's only
        p.v[0, first, 0, 7, 3] = float("nan")
    else:
        p.v_scale[0, last, 0, (p.lens[0] - 1) % 16] = float("inf")
        p.v_scale[0, first, 0, 3] = float("nan")
    lists[:, :, 0] = np.where(lists[:, :, 0] == 0, -1, lists[:, :, 0])
    got = attend(p, lists, causal=True).double().numpy()
    has = [t for t, _, at in p.columns() if at == p.lens[0] - 1 and (lists[t] == at // 16).any()]
    for t in range(p.tokens):
        assert np.isfinite(got[:, t]).all() == (t not in has), t
    lists[:, :, 0] = 0
    got = attend(p, lists)
    assert got.isnan().any(0).all()
    # keys: NaN and infinite scores, and scores of -inf alone
    p = Long(news, [200], 4, 1, 64, 16, cache, seed=10)
    lists = random_lists(p, 13)
    lists[:, :, 0] = 0
    (p.k if cache == "bf16" else p.k_scale)[0, p.table[0, 0], 0, 2] = float("nan")
    assert attend(p, lists).isnan().all()
    if cache == "bf16":
        p = Long(news, [200], 4, 1, 64, 16, seed=11)
        p.q.abs_()
        p.k[0, p.table[0, 0], 0] = -float("inf")
        assert attend(p, np.zeros((p.tokens, 1, 40), np.int32)).isnan().all()


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("scale", [1e-45, 1e-9, 3e38])
def test_scales_of_any_size(scale, cache):
    """The smallest weigh all alike; with zero queries the largest do too."""
    p = Long([1, 5], [300, 40], 4, 2, 64, 32, cache, seed=12)
    if scale > 1:
        p.q.zero_()
    lists = random_lists(p, 8)
    check(p, lists, scale=scale)


def test_weights_of_all_pages_are_those_of_plain_attention():
    """With lists of all pages both kinds of attention compute the same; other streams, replays of a graph."""
    p = Long([1, 1, 1], [500, 77, 1300], 8, 2, 128, 64, seed=13)
    cache, batch = p.on_device()
    lists = ints(np.tile(np.arange(p.width), (3, 2, 1)))
    how = sp.make_attend(8, 1, 128 ** -0.5, True, 0, "f32")
    q, a, b = p.q.cuda(), torch.empty((1024, 3), device="cuda"), torch.empty((1024, 3), device="cuda")
    work = torch.empty(sp.spmm_selected_work_bytes(cache, 3, how, p.width), dtype=torch.uint8, device="cuda")
    more = torch.empty(sp.spmm_attend_work_bytes(cache, 3, 3, how), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side_stream()):
        sp.spmm_cache_attend_selected(cache, 0, batch, q, 3, how, lists, p.width, a, 3, work, stream())
    for _ in range(3):
        q.normal_()
        graph.replay()
        sp.spmm_cache_attend(cache, 0, batch, q, 3, how, b, 3, more, stream())
        torch.cuda.synchronize()
        assert ((a - b).norm() <= 4e-3 * b.norm()).item()


def weigh(p, max_new=None, causal=True, window=0, decay=0.5, times=1, T=None):
    cache, batch = p.on_device()
    T = T or max(1, p.tokens)
    how = sp.make_weigh(p.q_heads, max_new or max(p.news + [1]), p.dim ** -0.5, causal, window, decay)
    work = torch.full((sp.spmm_weigh_work_bytes(cache, batch, T, how),), 255, dtype=torch.uint8, device="cuda")
    q = p.q.cuda()
    for _ in range(times):
        sp.spmm_cache_weigh(cache, p.layer, batch, q, T, how, work, stream())
    torch.cuda.synchronize()
    return p.dw.cpu().double().numpy()


def check_weights(p, max_new=None, causal=True, window=0, decay=0.5, **kw):
    got = weigh(p, max_new, causal, window, decay, **kw)
    want, added = p.weights_wanted(max_new or max(p.news + [1]), p.dim ** -0.5, causal, window, decay)
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= 3e-4 * added + 2.0 ** -22 * np.abs(want)) | (got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_weights_of_one_token_each(q_heads, kv_heads, dim, page, cache):
    check_weights(Long([1] * 7, [0, 1, 15, 16, 63, 200, 1000], q_heads, kv_heads, dim, page, cache, layers=2, layer=1, seed=21))


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim", HEADS[:4])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 23), (False, 40), (True, 1)])
@pytest.mark.parametrize("max_new", [1, 16, 1000])
def test_weights_of_chunks(q_heads, kv_heads, dim, causal, window, max_new, cache):
    check_weights(Long([3, 0, 70, 17, 1], [0, 5, 31, 130, 64], q_heads, kv_heads, dim, 32, cache, lead=2, seed=22), max_new, causal, window)


@pytest.mark.parametrize("news, pasts", [([300], [0]), ([129, 7], [500, 3000]), ([1], [9000]), ([1] * 90, [100] * 90), ([33, 1], [5000, 2])])
def test_weights_of_long_ones(news, pasts):
    check_weights(Long(news, pasts, 4, 2, 64, 16, seed=23))
    check_weights(Long(news, pasts, 2, 1, 128, 128, "s8", seed=24), max_new=20)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim", [(32, 8, 64), (32, 8, 128), (32, 8, 80), (160, 8, 16)])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 300)])
def test_weights_of_many_keys_and_columns(q_heads, kv_heads, dim, causal, window, cache):
    """Enough blocks of keys for the larger ones, and several of them for a workgroup."""
    check_weights(Long([5, 0, 6, 5, 5, 40, 5, 5], [900, 17, 1100, 3, 640, 1023, 511, 70], q_heads, kv_heads, dim, 64, cache, seed=31), causal=causal, window=window)
    if dim == 64:
        check_weights(Long([6] * 8, [250 * i + 1700 for i in range(8)], q_heads, kv_heads, dim, 64, cache, seed=32), causal=causal, window=window)


@pytest.mark.parametrize("decay", [0.0, 0.25, 1.0])
def test_what_stays_of_earlier_weights(decay):
    p = Long([2, 0, 5], [100, 30, 0], 4, 2, 64, 16, seed=25)
    p.weight[0, p.table[2, 0]] = float("nan")       # new tokens' weights need no initialisation
    p.weight[0, p.table[0, 102 // 16], :, (102 % 16):] = float("nan")
    if decay == 0.0:
        p.weight[0, p.table[0, 0], :, 3] = float("nan")     # nothing stays of it
        want = p.weight.clone()
        want[0, p.table[0, 0], :, 3] = 1.0
        got = weigh(p, decay=0.0)
        p.weight = want
        ref, added = p.weights_wanted(5, 64 ** -0.5, decay=0.0)
        fine = ~np.isnan(ref)
        assert (np.abs(got - ref)[fine] <= 3e-4 * added[fine] + 2.0 ** -22 * np.abs(ref[fine])).all()
    else:
        check_weights(p, decay=decay)


@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_rows_that_see_nothing(causal):
    p = Long([4, 1, 40], [20, 0, 0], 2, 1, 64, 16, seed=26)
    p.lens = [2, 0, 7]
    check_weights(p, causal=causal)
    check_weights(p, causal=causal, window=(1 << 31) - 1)
    check_weights(Long([3], [60], 2, 1, 64, 16, seed=27, width=2), causal=causal)
    p = Long([5, 9], [10, 30], 2, 1, 64, 16, seed=28)
    got = weigh(p, T=3)     # fewer columns than the batch says: those of the others are not there
    assert np.isfinite(got).all()


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("new", [1, 30])
def test_weights_of_what_is_not_finite(new, cache):
    p = Long([new, 2], [100, 40], 2, 2, 64, 16, cache, seed=29)
    x = p.k if cache == "bf16" else p.k_scale
    x[0, p.table[0, 0], 0, 2] = float("nan")
    x[0, p.table[1, 0], 1, 2] = float("inf")        # (8 bits: a score of NaN; bfloat16: infinities of either sign, so NaN)
    got = weigh(p)
    j = np.arange(100 + new)
    assert np.isnan(got[0, p.table[0, j // 16], 0, j % 16]).all() and np.isfinite(got[0, p.table[0, j // 16], 1, j % 16]).all()
    j = np.arange(42)
    assert np.isnan(got[0, p.table[1, j // 16], 1, j % 16]).all() and np.isfinite(got[0, p.table[1, j // 16], 0, j % 16]).all()


def test_weights_do_not_change_from_call_to_call_and_replay():
    p = Long([1, 40, 3], [700, 900, 0], 8, 2, 64, 32, seed=30)
    first = weigh(p)
    for _ in range(3):
        assert (weigh(p) == first).all()
    cache, batch = p.on_device()
    how = sp.make_weigh(8, 40, 0.125, True, 0, 0.5)
    work = torch.empty(sp.spmm_weigh_work_bytes(cache, batch, p.tokens, how), dtype=torch.uint8, device="cuda")
    q = p.q.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side_stream()):
        sp.spmm_cache_weigh(cache, 0, batch, q, p.tokens, how, work, stream())
    twice = p.weight.cuda()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        got = p.dw.clone()
        p.dw.copy_(twice)
        sp.spmm_cache_weigh(cache, 0, batch, q, p.tokens, how, work, stream())
        torch.cuda.synchronize()
        assert torch.equal(got, p.dw)
        twice = got
