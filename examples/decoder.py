"""A small decoder's attention layers in 8 bits, on sparse weights and a paged cache: prompts in chunks, then beams.

Every layer is  spmm_run (stacked Q/K/V weights, binary32)  ->  spmm_cache_append (norms, rotation, pages)  ->
spmm_cache_attend (u8)  ->  spmm_run (output projection, quantised for the next layer).  Activations stay on the device in the
library's order, rows = features; between steps spmm_cache_fork moves the beams on and spmm_cache_compact tidies the pool.
Weights are random and pruned in 4x1 blocks; there is no feed-forward part and no vocabulary, a step's input is random codes.

    python examples/decoder.py          runs it and prints the steps' times
"""
from __future__ import annotations

import os
import sys
import time

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2306_16601_amd as sp  # noqa: E402

HIDDEN, HEADS, KV_HEADS, DIM, LAYERS, PAGE = 768, 12, 4, 64, 3, 32
SPARSITY = 0.8
ZERO, SCALE = 128, 0.02       # of activations between layers, unsigned 8 bits


def pruned(rng, rows, cols):
    """int8 weight with 4x1 blocks (4 rows, one column) kept at random."""
    keep = rng.random((rows // 4, cols)) >= SPARSITY
    return (rng.integers(-127, 128, (rows, cols)) * np.repeat(keep, 4, axis=0)).astype(np.int8)


class Decoder:
    def __init__(self, pages: int, cache="bf16", seed: int = 0):
        rng = np.random.default_rng(seed)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()      # noqa: E731
        self.qkv_rows = (HEADS + 2 * KV_HEADS) * DIM
        unit = 1.0 / (73.0 * 1.0 * (HIDDEN * (1 - SPARSITY)) ** 0.5)        # results of about 1
        self.qkv = [sp.spmm_pack(pruned(rng, self.qkv_rows, HIDDEN)) for _ in range(LAYERS)]
        self.out = [sp.spmm_pack(pruned(rng, HIDDEN, HEADS * DIM)) for _ in range(LAYERS)]
        qkv_scale, out_scale = dev(np.full(self.qkv_rows, unit, np.float32)), dev(np.full(HIDDEN, 2 * unit, np.float32))
        self.to_qkv = sp.make_epilogue(qkv_scale, SCALE, ZERO, out_type="f32")
        self.to_hidden = sp.make_epilogue(out_scale, SCALE, ZERO, out_type="u8", out_scale=SCALE, out_zero_point=ZERO)
        weights = [dev(rng.uniform(0.5, 1.5, DIM).astype(np.float32)) for _ in range(2)]
        self.how = sp.make_append(HEADS, "f32", 1.0, 0, weights[0], weights[1], 1e-6, sp.make_rope(4096, DIM).cuda(), False)
        shape = (LAYERS, pages, KV_HEADS)
        kind = torch.int8 if cache == "s8" else torch.bfloat16
        scales = [torch.empty((*shape, PAGE), device="cuda") if cache == "s8" else None for _ in range(2)]
        self.cache = sp.make_cache(torch.empty((*shape, PAGE, DIM), dtype=kind, device="cuda"), torch.empty((*shape, DIM, PAGE), dtype=kind, device="cuda"), *scales)
        self.work = torch.empty(sp.spmm_cache_work_bytes(self.cache, 256), dtype=torch.uint8, device="cuda")
        self.info = torch.empty(4, dtype=torch.int32, device="cuda")

    def step(self, x, new, table, kv_len):
        """x [HIDDEN][T] u8: the new tokens of all sequences, new[b] each, the last ones of kv_len[b] -> the last layer's
        output in u8, and the attention of the last layer in binary32, [HEADS * DIM][T]."""
        T, stream = x.shape[1], torch.cuda.current_stream().cuda_stream
        start = torch.tensor(np.concatenate(([0], np.cumsum(new))).astype(np.int32), device="cuda")
        batch = sp.make_batch(start, kv_len, table)
        qkv = torch.empty((self.qkv_rows, T), device="cuda")
        q = torch.empty((T, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
        mid = torch.empty((HEADS * DIM, T), dtype=torch.uint8, device="cuda")
        exact = torch.empty((HEADS * DIM, T), device="cuda")
        attend = sp.make_attend(HEADS, max(new), DIM ** -0.5, True, 0, "u8", SCALE, ZERO)
        look = sp.make_attend(HEADS, max(new), DIM ** -0.5, True, 0, "f32")
        work = torch.empty(sp.spmm_attend_work_bytes(self.cache, len(new), T, attend), dtype=torch.uint8, device="cuda")
        for i in range(LAYERS):
            sp.spmm_run(self.qkv[i], x, T, T, self.to_qkv, qkv, T, stream)
            sp.spmm_cache_append(self.cache, i, batch, qkv, T, T, self.how, q, stream)
            sp.spmm_cache_attend(self.cache, i, batch, q, T, attend, mid, T, work, stream)
            if i == LAYERS - 1:
                sp.spmm_cache_attend(self.cache, i, batch, q, T, look, exact, T, work, stream)
            x = torch.empty((HIDDEN, T), dtype=torch.uint8, device="cuda")
            sp.spmm_run(self.out[i], mid, T, T, self.to_hidden, x, T, stream)
        return x, exact

    def fork(self, table, kv_len, parent, keep, want):
        """The sequences' next generation: (table, lengths)."""
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")      # noqa: E731
        table_out, len_out = torch.empty((len(parent), table.shape[1]), dtype=torch.int32, device="cuda"), torch.empty(len(parent), dtype=torch.int32, device="cuda")
        sp.spmm_cache_fork(self.cache, table, kv_len, ints(parent), ints(keep), ints(want), table_out, len_out, self.info, self.work, torch.cuda.current_stream().cuda_stream)
        return table_out, len_out

    def compact(self, table):
        sp.spmm_cache_compact(self.cache, table, table, self.info, self.work, torch.cuda.current_stream().cuda_stream)

    def close(self):
        for h in self.qkv + self.out:
            sp.spmm_destroy(h)


def columns(seqs):
    """Sequences of codes [HIDDEN][n] side by side."""
    return torch.from_numpy(np.concatenate(seqs, axis=1)).cuda()


def main(prompts=(70, 33), beams=4, steps=6, cache="bf16", tell=print):
    """Prompts in chunks of at most 40 tokens, then beams; returns every sequence's codes and what the last step attended to."""
    rng = np.random.default_rng(1)
    model = Decoder(pages=64, cache=cache)
    n, width = len(prompts), 8
    codes = [rng.integers(0, 256, (HIDDEN, p)).astype(np.uint8) for p in prompts]
    table, lens = torch.full((n, width), -1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    at = [0] * n
    while any(a < p for a, p in zip(at, prompts)):
        new = [min(40, p - a) for a, p in zip(at, prompts)]
        table, lens = model.fork(table, lens, list(range(n)), at, [a + c for a, c in zip(at, new)])
        began = time.perf_counter()
        model.step(columns([c[:, a:a + k] for c, a, k in zip(codes, at, new)]), new, table, torch.tensor([a + k for a, k in zip(at, new)], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        at = [a + k for a, k in zip(at, new)]
        lens = torch.tensor(at, dtype=torch.int32, device="cuda")
        tell("chunk of %s tokens: %.2f ms" % (new, 1e3 * (time.perf_counter() - began)))
    parent = [b for b in range(n) for _ in range(beams)]
    for step in range(steps):
        rows = len(parent)
        codes, at = [codes[p] for p in parent], [at[p] for p in parent]
        table, lens = model.fork(table, lens, parent, at, [a + 1 for a in at])
        if step % 3 == 2:
            model.compact(table)
        token = rng.integers(0, 256, (HIDDEN, rows)).astype(np.uint8)
        codes = [np.concatenate((c, token[:, j:j + 1]), axis=1) for j, c in enumerate(codes)]
        at = [a + 1 for a in at]
        lens = torch.tensor(at, dtype=torch.int32, device="cuda")
        began = time.perf_counter()
        _, last = model.step(torch.from_numpy(token).cuda(), [1] * rows, table, lens)
        torch.cuda.synchronize()
        used = model.info.cpu().tolist()
        tell("token %d of %d beams: %.2f ms, %d pages in use" % (step, rows, 1e3 * (time.perf_counter() - began), used[2]))
        parent = [j - j % beams + int(k) for j, k in enumerate(rng.integers(0, beams, rows))]
    model.close()
    return codes, last.cpu(), used


if __name__ == "__main__":
    main()
