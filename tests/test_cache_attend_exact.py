"""spmm_cache_attend on the device where its rounding is known: weights that are all 1, so that a token that is left out or counted twice
shows among thousands, and 8-bit caches at what binary16 operands leave."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import Problem
from test_cache_attend import attend

pytestmark = pytest.mark.gpu


def whole_numbers(p):
    """Values that are whole numbers (in 8 bits: codes, and one power of two as the scale), and zero queries."""
    p.q.zero_()
    r = np.random.default_rng(71)
    codes = torch.from_numpy(r.integers(-8, 9, tuple(p.v.shape))).to(p.v.dtype)
    if p.kind == "s8":
        p.v, p.v_scale = codes, torch.where(p.v_scale.isnan(), p.v_scale, torch.full_like(p.v_scale, 0.125))
    else:
        p.v = torch.where(p.v.isnan(), p.v, codes)


def means(p, causal, window):
    """Mean of the visible values, [q_heads * dim, tokens]."""
    out = np.zeros((p.q_heads, p.dim, p.tokens))
    values = p.v.double().transpose(3, 4).numpy()
    for b, n in enumerate(p.news):
        at = p.lens[b] - n + np.arange(n)
        for h in range(p.kv_heads if n else 0):
            v = p._rows(b, h, values, p.v_scale)
            sums = np.concatenate((np.zeros((1, p.dim)), np.cumsum(v, axis=0)))
            hi = np.where(at < 0, 0, np.minimum(at + 1, len(v)) if causal else len(v))
            lo = np.minimum(np.maximum(at - window + 1, 0), hi) if window else np.zeros_like(hi)
            y = (sums[hi] - sums[lo]) / np.maximum(hi - lo, 1)[:, None]
            out[h * p.group:(h + 1) * p.group, :, p.start[b]:p.start[b + 1]] = y.T
    return out.reshape(-1, p.tokens)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("causal, window", [(True, 0), (False, 0), (True, 777), (False, 2000)])
@pytest.mark.parametrize("news, pasts, heads", [
    ([1], [0], (1, 1, 64)), ([1, 1, 1], [1022, 63, 0], (4, 4, 64)), ([1, 3, 2, 1], [5000, 33333, 100, 8191], (8, 2, 128)), ([1, 0, 2], [70000, 5, 900], (2, 1, 80)),
    ([9, 1, 8], [1500, 4000, 0], (6, 2, 128)), ([40, 3, 33], [3000, 9000, 0], (4, 2, 128)), ([700, 130], [0, 2500], (2, 1, 64)), ([300], [5000], (4, 1, 96)),
    ([33] * 40, [1000] * 40, (16, 8, 64)), ([128] * 12, [500] * 12, (16, 8, 64))])
def test_every_visible_token_counts_once(news, pasts, heads, causal, window, page, cache):
    """Sums of whole numbers below 2^24 are exact in binary32, in any order; what is left is a reciprocal and a product, each off by
    at most a unit in the last place of binary32."""
    p = Problem(news, pasts, *heads, page, cache, seed=72)
    whole_numbers(p)
    got, ref = attend(p, causal=causal, window=window).double().numpy(), means(p, causal, window)
    bad = ~(np.abs(got - ref) <= 2.0 ** -22 * np.abs(ref))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])


@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("news, pasts, heads", [([1, 3, 2], [5000, 700, 0], (4, 2, 128)), ([1, 1], [900, 30], (4, 4, 64)), ([60, 300], [900, 0], (4, 2, 64)),
                                                ([250, 9], [40, 2000], (2, 1, 128)), ([40] * 40, [100] * 40, (8, 4, 80))])
def test_caches_of_8_bits_lose_what_binary16_does(news, pasts, heads, spread):
    """Queries, weights and, for many columns, keys and values are rounded to binary16: by 2^-11 of each, and in a subnormal by 2^-25 of the
    power of two that the largest was brought to.  Scores move by the former's share of sum |q k|, on both sides of the softmax."""
    p = Problem(news, pasts, *heads, 32, "s8", seed=73)
    p.q = (p.q.float() * 0.2).to(torch.bfloat16)
    if spread:      # scales over four orders of magnitude
        r = np.random.default_rng(74)
        for name in ("k_scale", "v_scale"):
            x = getattr(p, name)
            setattr(p, name, torch.where(x.isnan(), x, torch.from_numpy((0.04 * 10 ** r.uniform(-4, 0, tuple(x.shape))).astype(np.float32))))
    got = attend(p).double().numpy().reshape(p.q_heads, p.dim, -1)
    many = max(news) * p.group > 32
    half, sub, scale = 2.0 ** -11, 2.0 ** -25, p.dim ** -0.5
    keys, values = p.k.double().numpy(), p.v.double().transpose(3, 4).numpy()
    for b, n in enumerate(news):
        at = p.lens[b] - n + np.arange(n)[:, None]
        for h in range(p.q_heads):
            k, v = p._rows(b, h // p.group, keys, p.k_scale), p._rows(b, h // p.group, values, p.v_scale)
            sees = np.arange(len(k)) <= at
            t = slice(p.start[b], p.start[b + 1])
            q = p.q[t, h].double().numpy()
            w = np.where(sees, np.exp(np.where(sees, q @ k.T * scale, -np.inf) - np.where(sees, q @ k.T * scale, -np.inf).max(1, keepdims=True)), 0)
            l = w.sum(1, keepdims=True)
            move = sub * 2 * np.abs(q).max(1, keepdims=True) * np.abs(k).sum(1)
            if many:
                move = move + half * np.abs(q) @ np.abs(k).T + sub * np.abs(q).sum(1, keepdims=True) * 2 * np.nanmax(p.k_scale.numpy())
            move = np.where(sees, move, 0).max(1, keepdims=True) * scale
            tol = ((4 * half + 2 * move + 1e-4) * (w @ np.abs(v)) + (sub * 2 * np.nanmax(p.v_scale.numpy()) * (127 + 2 * many) * sees.sum(1, keepdims=True))) / l
            if many:        # (a value's own rounding, under weights that sum to 1)
                tol = tol + sub * 2 * np.nanmax(p.v_scale.numpy())
            bad = ~(np.abs(got[h, :, t] - (w @ v / l).T) <= tol.T)
            assert not bad.any(), (b, h, int(bad.sum()), np.argwhere(bad)[:5])
