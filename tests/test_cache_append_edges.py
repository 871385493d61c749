"""spmm_cache_append on the device with values that are not finite, or hardly more than zero, in both of its forms (heads of 64 dims,
and any others)."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import Problem

pytestmark = pytest.mark.gpu

TOKENS = 9


def append(x, dim, cache="s8", norm=False, rope=None, positions=None):
    """(queries, keys, values) as they are held, [tokens, heads, dim] each, and the scales of the latter, [tokens, heads]: two query heads
    on two, nine tokens behind five."""
    p = Problem([TOKENS], [5], 2, 2, dim, 16, cache, seed=51)
    c, batch = p.on_device()
    q = torch.empty((TOKENS, 2, dim), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(dim, device="cuda") if norm else None
    at = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    how = sp.make_append(2, "f32", 1.0, 0, w, w, 1e-6, None if rope is None else rope.cuda(), False, at)
    sp.spmm_cache_append(c, 0, batch, torch.from_numpy(x).cuda(), TOKENS, TOKENS, how, q, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    place = np.arange(5, 5 + TOKENS)
    page, off = p.table[0, place // 16], place % 16
    k, v = p.dk[0].float().cpu().numpy()[page, :, off], p.dv[0].float().cpu().numpy()[page, :, :, off]
    ks, vs = (None if s is None else s[0].cpu().numpy()[page, :, off] for s in (p.dks, p.dvs))
    return q.float().cpu().numpy(), k, v, ks, vs


def random(dim, seed=0):
    return np.random.default_rng(seed).standard_normal((6 * dim, TOKENS)).astype(np.float32)


def heads(x, dim):
    """keys and values of x, [tokens, heads, dim]"""
    y = x.reshape(6, dim, TOKENS).transpose(2, 0, 1)
    return y[:, 2:4], y[:, 4:]


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("positions", [None, [3, -1, 7, 8, 1 << 30, 0, 1, 2, 5]])
def test_positions_outside_the_table_give_nan_in_8_bits(positions, dim):
    """(Without positions of their own the tokens are at 5 .. 13.)"""
    _, k, v, ks, vs = append(random(dim), dim, norm=True, rope=sp.make_rope(8, dim), positions=positions)
    outside = np.array([not 0 <= at < 8 for at in (positions or range(5, 14))])
    assert outside.any() and not outside.all()
    assert (np.isnan(k * ks[..., None]) == outside[:, None, None]).all()
    assert np.isfinite(v * vs[..., None]).all()


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("norm", [True, False])
def test_what_is_not_finite_is_not_lost_in_8_bits(norm, odd, dim):
    """A token's head with such a value has a scale that is not finite, and none of its dims is; all others are as they were."""
    x = random(dim)
    x[2 * dim + 7, 1] = x[4 * dim + dim - 1, 3] = odd       # the first key head's, and the first value head's
    _, k, v, ks, vs = append(x, dim, norm=norm)
    clean = append(random(dim), dim, norm=norm)
    for got, scale, ref, ref_scale, token in ((k, ks, clean[1], clean[3], 1), (v, vs, clean[2], clean[4], 3)):
        with np.errstate(invalid="ignore"):
            assert not np.isfinite(got[token, 0] * scale[token, 0]).any()
        assert not np.isnan(odd) or np.isnan(scale[token, 0])
        others = np.ones(scale.shape, bool)
        others[token, 0] = False
        assert (got[others] == ref[others]).all() and (scale[others] == ref_scale[others]).all()


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("size", [1e-36, 2e-37, 1e-38, 1e-40, 1e-43])
def test_tiny_values_have_codes_of_their_own(size, dim):
    """Off by half a step of the scale, and by what binary32 holds of the scale itself (steps of 1.4e-45, for codes up to 127)."""
    x = (random(dim) * np.float32(size)).astype(np.float32)
    _, k, v, ks, vs = append(x, dim)
    for got, scale, ref in ((k, ks, heads(x, dim)[0]), (v, vs, heads(x, dim)[1])):
        ref = ref.astype(np.float64)
        scale = scale.astype(np.float64)[..., None]
        assert (np.abs(got * scale - ref) <= 0.501 * scale + 128 * 1.41e-45).all()
        assert (np.abs(got).max(-1) <= 127).all()
