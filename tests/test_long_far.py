"""The operators of long contexts where addresses pass 32 bits, on two streams at once, and in graphs that share scratch: the same bits as the same
problem close by and alone, which the operators' own tests compare with their definitions."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import side_stream
from long_reference import Long, ints, stream

pytestmark = pytest.mark.gpu

POOL = 70000        # pages of 128 tokens of 2 heads of 64 dims: the second layer's lie beyond 2^32 bytes, and 2^31 values


def problem(cache="bf16", seed=70):
    return Long([1, 40, 5], [700, 900, 0], 8, 2, 64, 128, cache, layers=2, layer=1, seed=seed)


class Run:
    """A problem's tensors, its pages moved up by `up` in a pool of `pages`, and what the calls write."""

    def __init__(self, p, pages=None, up=0, lds=None):
        pages = pages or p.pages
        self.p, self.up, self.lds = p, up, lds or p.width

        def part(x):
            if x is None:
                return None
            big = torch.zeros((x.shape[0], pages, *x.shape[2:]), dtype=x.dtype, device="cuda")
            big[:, up:up + p.pages] = x.cuda()
            return big
        self.parts = [part(x) for x in (p.k, p.v, p.k_scale, p.v_scale, p.bounds, p.weight)]
        self.cache = sp.make_cache(*self.parts)
        self.table = ints(np.where(p.table >= 0, p.table + up, -1))
        self.batch = sp.make_batch(ints(p.start), ints(p.lens), self.table)
        self.q, T = p.q.cuda(), p.tokens
        self.scores = torch.empty((T, 2, self.lds), device="cuda")
        self.lists = torch.full((T, 2, 3), -7, dtype=torch.int32, device="cuda")
        self.out = torch.full((8 * 64, T), 5.0, device="cuda")
        self.select, self.attend = sp.make_select(8, 3, 1, 1), sp.make_attend(8, 40, 0.125, out_type="f32")
        self.weigh, self.evict = sp.make_weigh(8, 40, 0.125, decay=0.5), sp.make_evict(4, 16, 300)
        self.kept = torch.full((2, 3, 2, 300), -7, dtype=torch.int32, device="cuda")
        self.lens_out = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.lens, self.keep = ints(p.lens), ints([300, 200, 5])
        need = max(sp.spmm_selected_work_bytes(self.cache, T, self.attend, 3), sp.spmm_weigh_work_bytes(self.cache, self.batch, T, self.weigh))
        self.work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")

    def read(self, at, work=None):
        T, work = self.p.tokens, self.work if work is None else work
        sp.spmm_cache_bounds(self.cache, 1, self.batch, T, at)
        sp.spmm_cache_score(self.cache, 1, self.batch, self.q, T, self.select, self.scores, self.lds, at)
        sp.spmm_cache_select(self.cache, self.batch, self.scores, T, self.lds, self.select, self.lists, at)
        sp.spmm_cache_attend_selected(self.cache, 1, self.batch, self.q, T, self.attend, self.lists, 3, self.out, T, work, at)

    def add(self, at, work=None):
        sp.spmm_cache_weigh(self.cache, 1, self.batch, self.q, self.p.tokens, self.weigh, self.work if work is None else work, at)

    def cut(self, at):
        sp.spmm_cache_evict(self.cache, self.table, self.lens, self.keep, self.evict, self.table, self.lens_out, self.kept, at)

    def all(self, at):
        self.read(at)
        self.add(at)
        self.cut(at)

    def results(self):
        torch.cuda.synchronize()
        mine = [None if x is None else x[:, self.up:self.up + self.p.pages].clone() for x in self.parts]
        return [self.scores[:, :, :self.p.width].clone(), self.lists, self.out, self.kept, self.lens_out] + [x for x in mine if x is not None]


def same(a, b):
    kinds = {1: torch.int8, 2: torch.int16, 4: torch.int32}
    return all(torch.equal(x.contiguous().view(kinds[x.element_size()]), y.contiguous().view(kinds[y.element_size()])) for x, y in zip(a, b))


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_pages_beyond_32_bits(cache):
    p = problem(cache)
    near, far = Run(p), Run(p, POOL * (2 if cache == "s8" else 1), POOL * (2 if cache == "s8" else 1) - p.pages)
    near.all(stream())
    far.all(stream())
    assert same(near.results(), far.results())
    assert all(x is None or not x[:, :far.up].any() for x in far.parts[4:])


def test_scores_beyond_32_bits():
    """Rows of scores a billion numbers apart."""
    p = Long([3], [300], 4, 1, 64, 16, seed=71)
    cache, batch = p.on_device()
    how, q = sp.make_select(4, 5), p.q.cuda()
    got = []
    for lds in (p.width, 1 << 30):
        scores, lists = torch.empty((3, 1, lds), device="cuda"), torch.full((3, 1, 5), -7, dtype=torch.int32, device="cuda")
        sp.spmm_cache_score(cache, 0, batch, q, 3, how, scores, lds, stream())
        sp.spmm_cache_select(cache, batch, scores, 3, lds, how, lists, stream())
        torch.cuda.synchronize()
        got.append((scores[:, :, :p.width].clone(), lists))
        del scores
    assert same(*got)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_two_streams_at_once(cache):
    first = [Run(problem(cache, 72 + i)) for i in range(2)]
    for r in first:
        r.all(stream())
    want = [r.results() for r in first]
    for _ in range(3):
        runs = [Run(problem(cache, 72 + i)) for i in range(2)]
        torch.cuda.synchronize()
        for r, at in zip(runs, (stream(), side_stream().cuda_stream)):
            r.all(at)
        assert all(same(r.results(), w) for r, w in zip(runs, want))


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_graphs_that_share_scratch(cache):
    a, b = Run(problem(cache, 74)), Run(problem(cache, 75))
    shared = torch.empty(max(a.work.numel(), b.work.numel()), dtype=torch.uint8, device="cuda")
    alone = [Run(problem(cache, 74)), Run(problem(cache, 75))]
    graphs = []
    torch.cuda.synchronize()
    for r in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side_stream()):
            now = torch.cuda.current_stream().cuda_stream
            r.read(now, shared)
            r.add(now, shared)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        for r in alone:
            r.read(stream())
            r.add(stream())
        shared.fill_(255)
        assert same(a.results(), alone[0].results()) and same(b.results(), alone[1].results())
