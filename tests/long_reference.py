"""The operators of long contexts from their definition, in 64 bits on the host, and the calls that tests make of them (test infrastructure)."""
import numpy as np
import torch

import paper_2306_16601_amd as sp
from cache_reference import Problem

OUT = {"f32": torch.float32, "bf16": torch.bfloat16, "s8": torch.int8, "u8": torch.uint8}
POISON = 77


def ints(values):
    return torch.tensor(np.ascontiguousarray(values), dtype=torch.int32, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


class Long(Problem):
    """A problem whose cache has bounds and weights: bounds of the pages as append would leave them, weights at random."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        shape = (self.layers, self.pages, self.k.shape[2])
        x = torch.from_numpy(self.rng.standard_normal((*shape, 2, self.dim), np.float32))
        self.bounds = torch.stack((x.amax(3), x.amin(3)), 3).to(torch.bfloat16)
        self.weight = torch.from_numpy(np.exp(self.rng.standard_normal((*shape, self.page), np.float32)))

    def on_device(self):
        self.dk, self.dv, self.db, self.dw = self.k.cuda(), self.v.cuda(), self.bounds.cuda(), self.weight.cuda()
        self.dks, self.dvs = (None if x is None else x.cuda() for x in (self.k_scale, self.v_scale))
        self.cache = sp.make_cache(self.dk, self.dv, self.dks, self.dvs, self.db, self.dw)
        self.batch = sp.make_batch(ints(self.start), ints(self.lens), ints(self.table))
        return self.cache, self.batch

    def held(self, b):
        """Tokens of a sequence that its table names."""
        return max(0, min(self.lens[b], self.width * self.page))

    def columns(self):
        """(column, sequence, first token that it sees, last one): of every sequence's columns."""
        for b, n in enumerate(self.news):
            for i in range(n):
                t = int(self.start[b]) + i
                if 0 <= t < self.tokens:
                    yield t, b, self.lens[b] - n + i

    def span(self, b, at, causal=True, window=0):
        n = self.held(b)
        if at < 0 or n == 0:
            return 0, -1
        return (min(max(0, at - window + 1), n) if window else 0), (min(at, n - 1) if causal else n - 1)

    def pages_seen(self, b, at, causal=True, window=0):
        lo, hi = self.span(b, at, causal, window)
        return (lo // self.page, hi // self.page) if lo <= hi else (1, 0)

    # ---- bounds

    def bounds_wanted(self):
        want = self.bounds.double().clone()
        for b, n in enumerate(self.news):
            length, past = self.held(b), self.lens[b] - n
            if n <= 0 or past >= length:
                continue
            for i in range(max(0, past) // self.page, -(-length // self.page)):
                page = self.table[b, i]
                if not 0 <= page < self.pages:
                    continue
                for h in range(self.k.shape[2]):
                    x = self.keys(b, h)[i * self.page:min(length, (i + 1) * self.page)]
                    both = np.stack((x.max(0), x.min(0)))
                    both[:, ~(np.abs(x) <= np.finfo(np.float32).max).all(0)] = np.nan      # (in binary32, as the cache's values are)
                    want[self.layer, page, h] = torch.from_numpy(both)
        return want

    # ---- score

    def scores_wanted(self, causal=True, window=0):
        """(scores, sums of magnitudes), NaN magnitudes where no column's are; [tokens, heads, width]"""
        shape = (max(1, self.tokens), self.k.shape[2], self.width)
        want, mag = np.full(shape, -np.inf), np.zeros(shape)
        mine = np.zeros(shape[0], bool)
        for t, b, at in self.columns():
            mine[t] = True
            lo, hi = self.pages_seen(b, at, causal, window)
            for h in range(shape[1]):
                limits = self.bounds[self.layer, self.table[b, lo:hi + 1], h].double().numpy()
                q = self.q[t, h * self.group:(h + 1) * self.group].double().numpy()[:, None]
                x = np.where(q > 0, q * limits[None, :, 0], q * limits[None, :, 1])
                want[t, h, lo:hi + 1] = x.sum(-1).max(0)
                mag[t, h, lo:hi + 1] = np.abs(x).sum(-1).max(0)
        return want, mag, mine

    # ---- select

    def lists_wanted(self, scores, pages, first, last, causal=True, window=0):
        want = np.full((max(1, self.tokens), scores.shape[1], pages), POISON, np.int32)
        for t, b, at in self.columns():
            lo, hi = self.pages_seen(b, at, causal, window)
            for h in range(scores.shape[1]):
                want[t, h] = chosen(scores[t, h], lo, hi, pages, first, last)
        return want

    # ---- attention over lists

    def selected_wanted(self, lists, scale, causal=True, window=0):
        out = np.full((self.q_heads, self.dim, max(1, self.tokens)), np.nan)
        mag, rows = out.copy(), {}
        for t, b, at in self.columns():
            lo, hi = self.span(b, at, causal, window)
            for h in range(self.q_heads):
                kv = h // self.group
                if (b, kv) not in rows:
                    rows[b, kv] = self.keys(b, kv), self.values(b, kv)
                k, v = rows[b, kv]
                j = np.concatenate([np.arange(i * self.page, (i + 1) * self.page) for i in lists[t, kv] if 0 <= i < self.width] or [np.zeros(0, int)]).astype(int)
                j = j[(j >= lo) & (j <= hi)]
                if not len(j):
                    out[h, :, t] = mag[h, :, t] = 0
                    continue
                s = k[j] @ self.q[t, h].double().numpy() * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[h, :, t], mag[h, :, t] = p @ v[j], p @ np.abs(v[j])
        return out.reshape(-1, max(1, self.tokens)), mag.reshape(-1, max(1, self.tokens))

    # ---- weigh

    def weights_wanted(self, max_new, scale, causal=True, window=0, decay=1.0):
        """(weights, what was added to each)"""
        want, added = self.weight.double().numpy().copy(), np.zeros(self.weight.shape)
        for b, n in enumerate(self.news):
            length = self.held(b)
            if n <= 0:
                continue
            past = self.lens[b] - n
            j = np.arange(length)
            pages, off = self.table[b, j // self.page], j % self.page
            for h in range(self.k.shape[2]):
                w = np.where(j < past, decay * want[self.layer, pages, h, off], 0.0)
                a = np.zeros(length)
                k = self.keys(b, h)
                for i in range(max(0, n - max_new), n):
                    t = int(self.start[b]) + i
                    lo, hi = self.span(b, past + i, causal, window)
                    if not 0 <= t < self.tokens or hi < lo:
                        continue
                    for head in range(h * self.group, (h + 1) * self.group):
                        s = k[lo:hi + 1] @ self.q[t, head].double().numpy() * scale
                        p = np.exp(s - s.max())
                        a[lo:hi + 1] += p / p.sum()
                want[self.layer, pages, h, off], added[self.layer, pages, h, off] = w + a, a
        return want, added


def order_of(x):
    """Highest first, of equal ones the earlier; NaN above all, -0 like 0."""
    x = np.where(np.isnan(x), np.inf, x + 0.0), np.isnan(x)
    return sorted(range(len(x[0])), key=lambda i: (not x[1][i], -x[0][i], i))


def chosen(scores, lo, hi, pages, first, last):
    """The list of one column and head."""
    n = max(0, hi - lo + 1)
    if n <= pages:
        ids = list(range(lo, lo + n))
    else:
        middle = np.asarray(scores[lo + first:hi + 1 - last], dtype=np.float64)
        best = order_of(middle)[:pages - first - last]
        ids = list(range(lo, lo + first)) + sorted(lo + first + i for i in best) + list(range(hi + 1 - last, hi + 1))
    return ids + [-1] * (pages - len(ids))


def kept_of(weights, n, first, recent):
    """The tokens that stay, of one row and head."""
    first = min(first, n)
    recent = min(recent, n - first)
    middle = weights[first:len(weights) - recent]
    best = order_of(np.asarray(middle, dtype=np.float64))[:n - first - recent]
    return list(range(first)) + sorted(first + i for i in best) + list(range(len(weights) - recent, len(weights)))
