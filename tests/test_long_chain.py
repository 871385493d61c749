"""The operators of long contexts one after the other, as a server would call them: prompts are read in chunks, their keys' bounds taken and
their attention added up, the contexts cut down, and new tokens read lists of the pages that are left.

Each step is compared with its definition for what the steps before left in the cache.  Tolerances are those of the operators' own tests."""
import copy
import os
import sys

import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import side_stream
from long_reference import Long, ints, kept_of, stream

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu

Q_HEADS, KV_HEADS, DIM, PAGE, LAYERS, WIDTH, PAGES = 8, 2, 64, 16, 2, 16, 40


class Server:
    def __init__(self, cache, seed):
        self.r = np.random.default_rng(seed)
        shape, kind = (LAYERS, PAGES, KV_HEADS), torch.int8 if cache == "s8" else torch.bfloat16
        full = lambda *s: torch.full((*shape, *s), float("nan"), device="cuda")     # noqa: E731
        self.k, self.v = (torch.zeros((*shape, *s), dtype=kind, device="cuda") for s in ((PAGE, DIM), (DIM, PAGE)))
        self.ks, self.vs = (full(PAGE) if cache == "s8" else None for _ in range(2))
        self.bounds, self.weight = full(2, DIM).to(torch.bfloat16), full(PAGE)
        self.cache = sp.make_cache(self.k, self.v, self.ks, self.vs, self.bounds, self.weight)
        self.work = torch.empty(sp.spmm_cache_work_bytes(self.cache, 16), dtype=torch.uint8, device="cuda")
        self.info = torch.empty(4, dtype=torch.int32, device="cuda")
        self.rope = sp.make_rope(1024, DIM).cuda()

    def fork(self, table, lens, parent, keep, want):
        out, lens_out = torch.empty((len(parent), WIDTH), dtype=torch.int32, device="cuda"), torch.empty(len(parent), dtype=torch.int32, device="cuda")
        sp.spmm_cache_fork(self.cache, table, lens, ints(parent), ints(keep), ints(want), out, lens_out, self.info, self.work, stream())
        assert self.info.cpu().tolist()[0] == 0
        return out

    def batch(self, news, lens, table):
        start = np.concatenate(([0], np.cumsum(news)))
        return sp.make_batch(ints(start), ints(lens), table)

    def append(self, layer, batch, T, positions):
        x = torch.from_numpy(self.r.standard_normal(((Q_HEADS + 2 * KV_HEADS) * DIM, T), np.float32)).cuda()
        q = torch.empty((T, Q_HEADS, DIM), dtype=torch.bfloat16, device="cuda")
        how = sp.make_append(Q_HEADS, rope=self.rope, positions=positions)
        sp.spmm_cache_append(self.cache, layer, batch, x, T, T, how, q, stream())
        return q

    def as_it_is(self, layer, news, lens, table, q=None):
        """The cache of this moment, as a problem whose definitions can be computed."""
        torch.cuda.synchronize()
        p = copy.copy(Long([1], [0], Q_HEADS, KV_HEADS, DIM, PAGE))
        p.layers, p.layer, p.pages, p.width, p.news, p.lens = LAYERS, layer, PAGES, WIDTH, list(news), list(lens)
        p.start = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
        p.tokens, p.table, p.q = int(p.start[-1]), table.cpu().numpy(), None if q is None else q.cpu()
        p.k, p.v, p.bounds, p.weight = self.k.cpu(), self.v.cpu(), self.bounds.cpu(), self.weight.cpu()
        p.k_scale, p.v_scale = (None if x is None else x.cpu() for x in (self.ks, self.vs))
        p.kind = "bf16" if self.ks is None else "s8"
        return p


def check_bounds(s, p):
    want = p.bounds_wanted()
    got = s.bounds.cpu().double()
    tol = (2.0 ** -8 + 2.0 ** -24) * want.abs() if p.kind == "s8" else 0 * want
    assert ((got - want).abs() <= tol)[~want.isnan()].all() and (got.isnan() == want.isnan()).all()


def keys_of(p, b, layer, j):
    """Keys, values (and scales) of tokens j of a row, as they are stored."""
    page, off = p.table[b, j // PAGE], j % PAGE
    parts = [p.k[layer, page, :, off], p.v[layer, page, :, :, off]]
    return parts + ([] if p.k_scale is None else [p.k_scale[layer, page, :, off], p.v_scale[layer, page, :, off]])


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_prompts_that_are_cut_down_and_read_by_lists(cache):
    s, lens = Server(cache, 1), [0, 0]
    table = torch.full((2, WIDTH), -1, dtype=torch.int32, device="cuda")
    how = sp.make_weigh(Q_HEADS, 8, DIM ** -0.5, decay=0.5)
    # prompts of 150 and 70 tokens, in two chunks
    for news in ([100, 40], [50, 30]):
        before, lens = lens, [n + k for n, k in zip(lens, news)]
        table = s.fork(table, ints(before), [0, 1], before, lens)
        batch, T = s.batch(news, lens, table), sum(news)
        for layer in range(LAYERS):
            q = s.append(layer, batch, T, None)
            old = s.as_it_is(layer, news, lens, table, q)
            sp.spmm_cache_bounds(s.cache, layer, batch, T, stream())
            work = torch.full((sp.spmm_weigh_work_bytes(s.cache, batch, T, how),), 255, dtype=torch.uint8, device="cuda")
            sp.spmm_cache_weigh(s.cache, layer, batch, q, T, how, work, stream())
            torch.cuda.synchronize()
            check_bounds(s, old)
            want, added = old.weights_wanted(8, DIM ** -0.5, decay=0.5)
            got, there = s.weight.cpu().double().numpy(), ~np.isnan(want)
            assert (np.isnan(got) == ~there).all()
            assert (np.abs(got - want)[there] <= 3e-4 * added[there] + 2.0 ** -22 * np.abs(want[there])).all()
    # the longer one is cut down to 64 tokens, in the pages that it has
    old = s.as_it_is(0, [1, 1], lens, table)
    lens_out, kept = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty((LAYERS, 2, KV_HEADS, 80), dtype=torch.int32, device="cuda")
    sp.spmm_cache_evict(s.cache, table, ints(lens), ints([64, 80]), sp.make_evict(4, 16, 80), table, lens_out, kept, stream())
    new = s.as_it_is(0, [1, 1], [64, 70], table)
    assert lens_out.cpu().tolist() == [64, 70]
    for layer in range(LAYERS):
        for h in range(KV_HEADS):
            page, off = old.table[0, np.arange(150) // PAGE], np.arange(150) % PAGE
            stay = np.array(kept_of(old.weight[layer, page, h, off].numpy(), 64, 4, 16))
            assert kept[layer, 0, h, :64].cpu().tolist() == stay.tolist()
            for x, y in zip(keys_of(old, 0, layer, stay), keys_of(new, 0, layer, np.arange(64))):
                assert torch.equal(x[:, h], y[:, h])
        for x, y in zip(keys_of(old, 1, layer, np.arange(70)), keys_of(new, 1, layer, np.arange(70))):
            assert torch.equal(x, y)
    # the pages behind are given back, and the bounds of the others taken anew
    at, lens = list(lens), [64, 70]
    table = s.fork(table, lens_out, [0, 1], lens, lens)
    assert (table[0, 4:] == -1).all() and s.info.cpu().tolist()[2] == 4 + 5
    whole = s.batch(lens, lens, table)
    for layer in range(LAYERS):
        sp.spmm_cache_bounds(s.cache, layer, whole, sum(lens), stream())
        check_bounds(s, s.as_it_is(layer, lens, lens, table))
    # new tokens go on counting from where the sequences were
    select, attend = sp.make_select(Q_HEADS, 3, 1, 1), sp.make_attend(Q_HEADS, 1, DIM ** -0.5, out_type="f32")
    for _ in range(3):
        before, lens = lens, [n + 1 for n in lens]
        table = s.fork(table, ints(before), [0, 1], before, lens)
        batch = s.batch([1, 1], lens, table)
        for layer in range(LAYERS):
            q = s.append(layer, batch, 2, ints(at))
            scores, lists = torch.empty((2, KV_HEADS, WIDTH), device="cuda"), torch.empty((2, KV_HEADS, 3), dtype=torch.int32, device="cuda")
            work = torch.full((sp.spmm_selected_work_bytes(s.cache, 2, attend, 3),), 255, dtype=torch.uint8, device="cuda")
            out = torch.empty((Q_HEADS * DIM, 2), device="cuda")

            def step():
                now = torch.cuda.current_stream().cuda_stream
                sp.spmm_cache_bounds(s.cache, layer, batch, 2, now)
                sp.spmm_cache_score(s.cache, layer, batch, q, 2, select, scores, WIDTH, now)
                sp.spmm_cache_select(s.cache, batch, scores, 2, WIDTH, select, lists, now)
                sp.spmm_cache_attend_selected(s.cache, layer, batch, q, 2, attend, lists, 3, out, 2, work, now)

            before_bounds = s.as_it_is(layer, [1, 1], lens, table, q)
            step()
            p = s.as_it_is(layer, [1, 1], lens, table, q)
            check_bounds(s, before_bounds)
            want, mag, _ = p.scores_wanted()
            got = scores.cpu().double().numpy()
            with np.errstate(invalid="ignore"):
                assert ((got == want) | (np.abs(got - want) <= 2 * DIM * 2.0 ** -23 * mag)).all()
            chosen = lists.cpu().numpy()
            assert (chosen == p.lists_wanted(got, 3, 1, 1)).all()
            ref, size = p.selected_wanted(chosen, DIM ** -0.5)
            assert (np.abs(out.cpu().double().numpy() - ref) <= (2.0 ** -8 + 1e-4) * size).all()
            # the same captured, and replayed with other things in between
            first = [x.clone() for x in (out, lists, scores, s.bounds)]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side_stream()):
                step()
            for _ in range(2):
                out.fill_(5.0), lists.fill_(-7), scores.fill_(9.0), work.fill_(255)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(x.nan_to_num(3.0), y.nan_to_num(3.0)) for x, y in zip(first, (out, lists, scores, s.bounds)))
        at = [n + 1 for n in at]


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_the_example_reads_lists(cache):
    """With lists of all pages and room for all tokens the contexts are whole: the same bound as in the example's other test."""
    import decoder
    codes, last, held = decoder.long_contexts(prompts=(150, 60), steps=3, room=256, listed=8, cache=cache, tell=lambda *a: None)
    assert held == [153, 63]
    whole = decoder.Decoder(pages=64, cache=cache)
    for b in range(2):
        n = codes[b].shape[1]
        table, lens = whole.fork(torch.full((1, 8), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), [-1], [0], [n])
        _, exact = whole.step(decoder.columns([codes[b]]), [n], table, torch.tensor([n], dtype=torch.int32, device="cuda"))
        ref, got = exact[:, -1].cpu().double(), last[:, b].double()
        assert (got - ref).norm() <= 0.05 * ref.norm()
    whole.close()


def test_the_example_cuts_contexts_down():
    import decoder
    codes, last, held = decoder.long_contexts(prompts=(150, 60), steps=3, room=96, listed=2, tell=lambda *a: None)
    assert [c.shape[1] for c in codes] == [153, 63] and held == [99, 63] and last.isfinite().all() and last.abs().sum() > 0
