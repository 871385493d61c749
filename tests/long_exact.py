"""How far attention over lists of pages may be from its definition where nothing is rounded to less than binary32 (test infrastructure).

With n visible tokens, D dims, A the largest sum of |q k| scale over the dims of a key, and unit roundings of 2^-24 (additions inside the matrix instruction are counted as 2^-23,
whichever way it rounds):
  scores      D additions of exact products: D 2^-23 A; queries beside 8-bit codes lose 2^-25 of the largest one: 2^-25 max |q| sum |k| scale; scale, the key's
              scale, the largest score and the exponent are rounded once each, to 2^-24 of at most 2 A log2(e) < 3 A: less than 2^-20 A together
  weights     twice that (their own error, and that of their sum), the exponential 2^-22; of 8-bit caches, in two terms of binary16, 2^-23 of themselves and
              2^-24 of the largest scale that they are multiplied beside: of the largest weight, which is part of the sum
  sums        3 n additions for products of three terms, n for the sum of the weights, 32 to join lanes, waves and parts: (4 n + 32) 2^-23
All but the losses beside the largest query and scale are relative to sum p |v|."""
import numpy as np


def limits(p, lists, scale, causal=True, window=0):
    """(result, how far off it may be), [q_heads * dim, tokens]; NaN in columns of no sequence."""
    out = np.full((p.q_heads, p.dim, max(1, p.tokens)), np.nan)
    tol, rows = out.copy(), {}
    for t, b, at in p.columns():
        lo, hi = p.span(b, at, causal, window)
        for h in range(p.q_heads):
            kv = h // p.group
            if (b, kv) not in rows:
                j = np.arange(p.held(b))
                scales = None if p.v_scale is None else p.v_scale.double().numpy()[p.layer, p.table[b, j // p.page], kv, j % p.page]
                rows[b, kv] = p.keys(b, kv), p.values(b, kv), scales
            k, v, scales = rows[b, kv]
            j = np.concatenate([np.arange(i * p.page, (i + 1) * p.page) for i in lists[t, kv] if 0 <= i < p.width] or [np.zeros(0, int)]).astype(int)
            j = j[(j >= lo) & (j <= hi)]
            if not len(j):
                out[h, :, t] = tol[h, :, t] = 0
                continue
            q = p.q[t, h].double().numpy()
            s = k[j] @ q * scale
            y = np.exp(s - s.max())
            w, n = y / y.sum(), len(j)
            off = (p.dim * 2.0 ** -23 + 2.0 ** -20) * (np.abs(k[j]) @ np.abs(q)).max() * scale
            lost = 0.0
            if scales is not None:
                off += 2.0 ** -25 * np.abs(q).max() * np.abs(k[j]).sum(1).max() * scale
                lost = 2.0 ** -24 * scales[j].max() * (np.abs(v[j]) / scales[j, None]).sum(0) / y.sum()
            out[h, :, t] = w @ v[j]
            tol[h, :, t] = (w @ np.abs(v[j])) * (2 * off + 2.0 ** -22 + 2.0 ** -23 + (4 * n + 32) * 2.0 ** -23) + lost
    return out.reshape(-1, max(1, p.tokens)), tol.reshape(-1, max(1, p.tokens))


def plant(p, what):
    """Puts into an 8-bit cache of one sequence: a scale that is not finite at the first token, and at the one in the middle of the new ones, which half of them see ("k nan",
    "k inf", "v nan", "v inf"), or value scales that differ by many powers of two from page to page ("spread", "wide")."""
    r = np.random.default_rng(9)
    if what in ("spread", "wide"):
        for i in range(p.width):
            if 0 <= p.table[0, i] < p.pages:
                p.v_scale[:, p.table[0, i]] *= 2.0 ** int(r.integers(-24, 25) if what == "spread" else r.choice((-120, 0, 100)))
        return
    part, value = what.split()
    scale = p.k_scale if part == "k" else p.v_scale
    for j in (0, p.lens[0] - p.news[0] + p.news[0] // 2):
        scale[p.layer, p.table[0, j // p.page], :, j % p.page] = float(value)


def compare(got, p, lists, scale, causal=True, window=0):
    """(number of results that are wrong, where): what is not finite in the definition has to be so, and nothing else."""
    with np.errstate(all="ignore"):
        ref, tol = limits(p, lists, scale, causal, window)
        mine = np.zeros(got.shape, bool)
        mine[:, [t for t, _, _ in p.columns()]] = True
        fine = np.isfinite(ref)
        bad = mine & ~np.where(fine, np.abs(got - ref) <= tol, ~np.isfinite(got))
    return int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3].tolist(), ref[bad][:3].tolist(), tol[bad][:3].tolist()


ODD = ["k nan", "k inf", "v nan", "v inf", "spread", "wide"]
# heads of queries and keys, dims, new tokens: lists with four waves each, and with one; 16, 4, 2 streams and one of the columns that heads leave free
MANY = [(4, 4, 64, 70), (4, 1, 128, 270), (10, 2, 48, 140), (16, 1, 96, 260), (6, 6, 64, 180), (16, 4, 64, 250), (32, 4, 32, 250), (64, 4, 128, 250)]


def share(p, groups):
    """Rows of each group (first row, others, pages) name the first one's first pages, as after a fork."""
    for first, others, pages in groups:
        for b in others:
            p.table[b, :pages] = p.table[first, :pages]


def shared_weights(p, max_new, scale, causal=True, window=0, decay=1.0, off=None):
    """(weights, what was added) where rows share pages: a token's weight fades once, or is new where it is that to one of the rows, and gets the shares of all.
    off: an array that how far each may be off is added to (the errors of scores, powers and sums as above; products are exact in both types of cache)."""
    held, fresh, added = (np.zeros(p.weight.shape, t) for t in (bool, bool, float))
    columns = np.zeros(p.weight.shape)
    for b, n in enumerate(p.news):
        length, past = p.held(b), p.lens[b] - n
        if n <= 0:
            continue
        j = np.arange(length)
        pages, slots = p.table[b, j // p.page], j % p.page
        held[p.layer, pages, :, slots] = True
        fresh[p.layer, pages[j >= past], :, slots[j >= past]] = True
        for h in range(p.k.shape[2]):
            k = p.keys(b, h)
            for i in range(max(0, n - max_new), n):
                lo, hi = p.span(b, past + i, causal, window)
                if hi < lo:
                    continue
                at = np.arange(lo, hi + 1)
                for head in range(h * p.group, (h + 1) * p.group):
                    s = k[at] @ p.q[int(p.start[b]) + i, head].double().numpy() * scale
                    y = np.exp(s - s.max())
                    added[p.layer, pages[at], h, slots[at]] += y / y.sum()
                    columns[p.layer, pages[at], h, slots[at]] += 1
                    if off is not None:
                        worst = (np.abs(k[at]) @ np.abs(p.q[int(p.start[b]) + i, head].double().numpy())).max() * scale
                        off[p.layer, pages[at], h, slots[at]] += y / y.sum() * (2 * (p.dim * 2.0 ** -23 + 2.0 ** -20) * worst + 2.0 ** -22 + (len(at) + 32) * 2.0 ** -23)
    if off is not None:
        off += (columns + 32) * 2.0 ** -23 * added + 2.0 ** -22 * p.weight.double().numpy() * held
    old = p.weight.double().numpy()
    return np.where(held, np.where(fresh, 0.0, decay * old) + added, old), added


# (new tokens, past, (first row, other rows, shared pages)): beams, a common prefix and one within it, rows that end inside a shared page or have nothing new
SHARED = [([1] * 5, [100, 100, 100, 37, 100], [(0, [1, 2, 4], 6)]), ([1, 2, 1, 0, 1, 3], [200, 150, 90, 200, 40, 10], [(0, [1, 2, 3], 4), (0, [4], 2)]),
          ([1, 1, 1], [63, 40, 70], [(0, [1, 2], 3)]), ([20, 5, 7], [100, 110, 64], [(0, [1, 2], 4)]), ([9, 40, 1, 12], [300, 900, 320, 17], [(0, [2], 18), (1, [3], 1)])]
