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


def by_kind(p, causal=True, window=0):
    """(result, sum of p |v|) as Problem.attention has them, for values that are not finite too: a sequence and a head at a time, their
    sums and NaN, +inf and -inf apart from each other."""
    out = np.full((p.q_heads, p.dim, p.tokens), np.nan)
    mag = out.copy()
    keys, values = p.k.double().numpy(), p.v.double().transpose(3, 4).numpy()
    for b, n in enumerate(p.news):
        at = p.lens[b] - n + np.arange(n)[:, None]
        for h in range(p.q_heads if n else 0):
            k, v = p._rows(b, h // p.group, keys, p.k_scale), p._rows(b, h // p.group, values, p.v_scale)
            j = np.arange(len(k))
            sees = np.broadcast_to(at >= 0, (n, len(k)))
            if causal:
                sees = sees & (j <= at)
            if window:
                sees = sees & (j > at - window)
            t = slice(p.start[b], p.start[b] + n)
            s = np.where(sees, p.q[t, h].double().numpy() @ k.T * p.dim ** -0.5, -np.inf)
            lost = (sees & ~(s < np.inf)).any(1) | (sees.any(1) & (s == -np.inf).all(1))       # (NaN, or nothing but -inf, among the scores)
            w = np.exp(s - np.where(np.isfinite(s), s, -1e300).max(1, keepdims=True))
            w /= np.maximum(w.sum(1, keepdims=True), 1e-300)
            w[lost] = 0
            plus, minus, nan = (sees.astype(float) @ kind(v) > 0 for kind in (np.isposinf, np.isneginf, np.isnan))
            finite = np.where(np.isfinite(v), v, 0)
            y = w @ finite
            y[plus], y[minus], y[nan | (plus & minus) | lost[:, None]] = np.inf, -np.inf, np.nan
            out[h, :, t], mag[h, :, t] = y.T, (w @ np.abs(finite)).T
    return out.reshape(-1, p.tokens), mag.reshape(-1, p.tokens)


def as_defined(p, got, causal=True, window=0):
    """Results that are not finite are NaN or infinities as the definition has them; the others are near it."""
    with np.errstate(invalid="ignore", over="ignore"):
        ref, mag = by_kind(p, causal, window)
    got = got.double().numpy()
    for kind in (np.isnan, np.isposinf, np.isneginf):
        bad = kind(got) != kind(ref)
        assert not bad.any(), (kind.__name__, int(bad.sum()), np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])
    fine = np.isfinite(ref)
    assert (np.abs(got[fine] - ref[fine]) <= (2.0 ** -8 + 1e-4) * mag[fine]).all()
    return ref


def test_the_definition_by_kind_is_the_definition():
    p = Problem([8, 1, 20], [150, 40, 3], 4, 2, 64, 16, seed=60)
    p.lens[2] = 9
    for causal, window in ((True, 0), (False, 0), (True, 30), (False, 5)):
        for x, y in zip(by_kind(p, causal, window), p.attention(p.dim ** -0.5, causal, window)):
            assert np.allclose(x, y, rtol=1e-12, atol=1e-12)


# new tokens and past of each sequence, table's width in pages of 16: heads that one workgroup takes, and runs that are joined; blocks
# of 128 columns in parts, and whole; the same of 256 columns (8 bits)
FORMS = {"whole": ([8, 1, 5], [150, 40, 0], None), "runs": ([8, 1, 5], [150, 40, 700], 90), "parts": ([70, 3, 260], [150, 40, 9], None),
         "blocks": ([34] * 150, [70] * 150, None), "wide parts": ([70, 3, 250], [150, 40, 9], None), "wide blocks": ([120] * 70, [70] * 70, None)}


def problem(form, cache, seed, dim=64):
    news, pasts, width = FORMS[form]
    p = Problem(news, pasts, 4, 2, dim, 16, cache, seed=seed, width=width)
    p.q = (p.q.float() * 0.3).to(torch.bfloat16)        # (weights that neither type of the products' operands loses)
    return p


def plant(p, what, b, at, value, dim=5):
    """A value of sequence b's token `at`, in one dim of its first head (of 8 bits: in the head's scale)."""
    page, off = int(p.table[b, at // 16]), at % 16
    if p.kind == "s8":
        (p.k_scale if what == "k" else p.v_scale)[0, page, 0, off] = value
    elif what == "k":
        p.k[0, page, 0, off, dim] = value
    else:
        p.v[0, page, 0, dim, off] = value


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 30)])
@pytest.mark.parametrize("odd", [NAN, INF, -INF])
def test_values_that_are_not_finite(odd, causal, window, form, cache):
    """In tokens that all of a sequence's new ones see, and in tokens that some see."""
    p = problem(form, cache, 61)
    for b in range(len(p.news)):
        plant(p, "v", b, (3, p.lens[b] // 2, p.lens[b] - p.news[b] // 2 - 1, p.lens[b] - 1)[b % 4], odd)
    ref = as_defined(p, attend(p, causal=causal, window=window), causal, window)
    assert not np.isfinite(ref).all()


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("odd", [NAN, INF, -INF])
@pytest.mark.parametrize("cache", CACHES)
def test_keys_that_are_not_finite(cache, odd, form):
    """(In 8 bits an infinite scale: dims of both signs, and so a score of NaN.)"""
    p = problem(form, cache, 63)
    for b, n in enumerate(p.lens):
        plant(p, "k", b, min(n - 1, 4 + n // 3), odd, dim=9)
    as_defined(p, attend(p))


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("seen_by_all, seen_by_some", [(INF, -INF), (-INF, INF), (NAN, INF), (INF, INF), (INF, NAN)])
@pytest.mark.parametrize("cache", CACHES)
def test_values_of_both_signs(cache, seen_by_all, seen_by_some, form):
    """An infinity that some columns see does not hide what they all see."""
    p = problem(form, cache, 62)
    for b, n in enumerate(p.lens):
        plant(p, "v", b, 2, seen_by_all)
        plant(p, "v", b, n - 1 - p.news[b] // 3, seen_by_some)
    as_defined(p, attend(p))


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("cache", CACHES)
def test_scores_of_nan_beside_infinite_values(cache, form):
    """A column with a score of NaN is NaN as a whole, whatever else it sees."""
    p = problem(form, cache, 64)
    for b, n in enumerate(p.lens):
        plant(p, "k", b, min(n - 1, 4 + n // 3), NAN, dim=9)
        plant(p, "v", b, n - 1 - p.news[b] // 3, INF)
    as_defined(p, attend(p))


@pytest.mark.parametrize("form", list(FORMS))
def test_nothing_but_scores_of_minus_infinity(form):
    """The softmax of nothing but -inf is NaN; 0 is the result only where nothing is visible."""
    p = problem(form, "bf16", 65)
    p.q[:, :, 9] = p.q[:, :, 9].abs() + 0.1
    for b, n in enumerate(p.lens):
        for at in range(n if b % 2 else min(n, p.lens[b] - p.news[b] + 2)):
            plant(p, "k", b, at, -INF, dim=9)
    ref = as_defined(p, attend(p))
    assert np.isnan(ref).any() and np.isfinite(ref).any()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("new", [1, 40, 300])
def test_the_largest_scale(new, cache):
    """log2(e) times it is beyond binary32; a zero query's scores are zero all the same."""
    p = Problem([new, 3], [77, 20], 4, 2, 64, 32, cache, seed=45)
    p.q.zero_()
    scale = 3.4e38
    got = attend(p, scale=scale).double().numpy()
    ref, mag = p.attention(scale)
    assert (np.abs(got - ref) <= (2.0 ** -8 + 1e-4) * mag).all()
