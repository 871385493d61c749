"""The paged cache's operators from their definition, token by token, in 64 bits on the host (test infrastructure)."""
import functools

import numpy as np
import torch


@functools.lru_cache(None)
def side_stream():
    """One stream for all these tests: streams share a few hardware queues in the order of their first use, and a test of the same
    process that looks at whether work on a stream of its own holds up the default one depends on how many came before."""
    return torch.cuda.Stream()


class Problem:
    """A cache of random pages and a batch over it; unused slots hold NaN (8-bit caches: scales of NaN)."""

    def __init__(self, news, pasts, q_heads, kv_heads, dim, page, cache="bf16", layers=1, layer=0, spare=3, seed=0, lead=0, width=None):
        r = np.random.default_rng(seed)
        self.news, self.pasts, self.q_heads, self.kv_heads, self.dim, self.page, self.kind = news, pasts, q_heads, kv_heads, dim, page, cache
        self.layers, self.layer, self.group = layers, layer, q_heads // kv_heads
        self.lens = [n + p for n, p in zip(news, pasts)]
        held = [max(0, -(-n // page)) for n in self.lens]
        self.pages = sum(held) + spare
        self.width = width or max(held + [1]) + 1
        order = r.permutation(self.pages)
        self.table, at = np.full((len(news), self.width), -1, np.int32), 0
        for b, n in enumerate(held):
            n = min(n, self.width)
            self.table[b, :n] = order[at:at + n]
            at += n
        self.start = np.concatenate(([0], np.cumsum(news))).astype(np.int32) + lead
        self.tokens = int(self.start[-1])
        shape = (layers, self.pages, kv_heads)
        k, v = (torch.from_numpy(r.standard_normal((*shape, page, dim), np.float32)) for _ in range(2))
        v = v.transpose(3, 4).contiguous()
        self.k_scale = self.v_scale = None
        stale = torch.ones((layers, self.pages, kv_heads, page), dtype=torch.bool)
        for b, n in enumerate(self.lens):
            for j in range(max(0, min(n, self.width * page))):
                stale[:, self.table[b, j // page], :, j % page] = False
        if cache == "s8":
            self.k, self.v = ((x * 40).round().clamp(-127, 127).to(torch.int8) for x in (k, v))
            self.k_scale, self.v_scale = (torch.from_numpy(r.uniform(0.01, 0.04, stale.shape).astype(np.float32)).masked_fill(stale, float("nan")) for _ in range(2))
        else:
            self.k = k.masked_fill(stale[..., None], float("nan")).to(torch.bfloat16)
            self.v = v.masked_fill(stale[..., None, :], float("nan")).to(torch.bfloat16)
        self.q = torch.from_numpy(r.standard_normal((max(1, self.tokens), q_heads, dim), np.float32) * 1.5).to(torch.bfloat16)
        self.rng = r

    def on_device(self):
        """cache, batch and the tensors behind them"""
        import paper_2306_16601_amd as sp
        self.dk, self.dv = self.k.cuda(), self.v.cuda()
        self.dks, self.dvs = (None if x is None else x.cuda() for x in (self.k_scale, self.v_scale))
        self.cache = sp.make_cache(self.dk, self.dv, self.dks, self.dvs)
        self.batch = sp.make_batch(torch.from_numpy(self.start).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), torch.from_numpy(self.table).cuda())
        return self.cache, self.batch

    def keys(self, b, h, k=None, scale=None):
        """All tokens' keys of a sequence and a head, float64 [tokens, dim]."""
        return self._rows(b, h, self.k.double().numpy(), self.k_scale)

    def values(self, b, h):
        return self._rows(b, h, self.v.double().transpose(3, 4).numpy(), self.v_scale)

    def _rows(self, b, h, x, scale):
        n = max(0, min(self.lens[b], self.width * self.page))
        j = np.arange(n)
        pages, off = self.table[b, j // self.page], j % self.page
        rows = x[self.layer, pages, h, off]
        return rows if scale is None else rows * scale.double().numpy()[self.layer, pages, h, off][:, None]

    def attention(self, scale, causal=True, window=0):
        """(result, sum of p |v|), float64 [q_heads * dim, tokens]; NaN where no sequence's column is."""
        out = np.full((self.q_heads, self.dim, max(1, self.tokens)), np.nan)
        mag = out.copy()
        for b, n in enumerate(self.news):
            for i in range(n):
                t, at = self.start[b] + i, self.lens[b] - n + i
                if t < 0 or t >= self.tokens:
                    continue
                for h in range(self.q_heads):
                    k, v = self.keys(b, h // self.group), self.values(b, h // self.group)
                    lo = max(0, at - window + 1) if window else 0
                    hi = 0 if at < 0 else min(at + 1, len(k)) if causal else len(k)
                    if hi <= lo:
                        out[h, :, t] = mag[h, :, t] = 0
                        continue
                    s = k[lo:hi] @ self.q[t, h].double().numpy() * scale
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[h, :, t], mag[h, :, t] = p @ v[lo:hi], p @ np.abs(v[lo:hi])
        return out.reshape(-1, max(1, self.tokens)), mag.reshape(-1, max(1, self.tokens))
