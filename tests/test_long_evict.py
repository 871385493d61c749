"""spmm_cache_evict on the device against its definition, and the page calls with all parts of a cache.  All of it is exact."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import side_stream
from long_reference import POISON, Long, ints, kept_of, stream

pytestmark = pytest.mark.gpu


class Row(Long):
    def __init__(self, lens, kv_heads, dim, page, cache="bf16", layers=2, seed=0, spare=0, width=None):
        super().__init__([1] * len(lens), [n - 1 for n in lens], kv_heads, kv_heads, dim, page, cache, layers=layers, seed=seed, spare=spare + sum(-(-n // page) for n in lens), width=width)

    def fresh(self, pages):
        """A table of other pages than the sequences', pages[b] each."""
        mine = set(self.table.flatten().tolist())
        free = [x for x in range(self.pages) if x not in mine]
        to = np.full_like(self.table, -1)
        for b, n in enumerate(pages):
            for i in range(min(n, self.width)):
                to[b, i] = free.pop()
        return to

    def evicted(self, keep, first, recent, most, to):
        """(kept, lengths, parts) by the header's rules"""
        parts = [x.clone() for x in (self.dk, self.dv, self.dks, self.dvs, self.dw) if x is not None]
        parts = [x.cpu() for x in parts]
        old = [x.clone() for x in parts]
        kept = np.full((self.layers, len(self.lens), self.k.shape[2], most), -1, np.int32)
        lens = [max(0, min(self.held(b), keep[b], most)) for b in range(len(self.lens))]
        for layer in range(self.layers):
            for b, n in enumerate(lens):
                j = np.arange(self.held(b))
                for h in range(self.k.shape[2]):
                    stay = kept_of(old[-1][layer, self.table[b, j // self.page], h, j % self.page].numpy(), n, first, recent)
                    kept[layer, b, h, :n] = stay
                    for slot, i in enumerate(stay):
                        page, off, at, o = self.table[b, i // self.page], i % self.page, to[b, slot // self.page], slot % self.page
                        if not 0 <= at < self.pages:
                            continue
                        for k, (x, y) in enumerate(zip(parts, old)):
                            if k == 1:
                                x[layer, at, h, :, o] = y[layer, page, h, :, off]
                            else:
                                x[layer, at, h, o] = y[layer, page, h, off]
        return kept, lens, parts


def evict(p, keep, first=2, recent=5, most=None, to=None, change=None, call_stream=None):
    if change:
        change(p.weight)
    cache, _ = p.on_device()
    most = most or max(max(keep), 1)
    table, table_to = ints(p.table), None
    to = p.table if to is None else to
    table_to = table if to is p.table else ints(to)
    want = p.evicted(keep, first, recent, most, to)
    kept = torch.full((p.layers, len(p.lens), p.k.shape[2], most), POISON, dtype=torch.int32, device="cuda")
    lens = torch.full((len(p.lens),), POISON, dtype=torch.int32, device="cuda")
    sp.spmm_cache_evict(cache, table, ints(p.lens), ints(keep), sp.make_evict(first, recent, most), table_to, lens, kept, stream())
    torch.cuda.synchronize()
    assert lens.cpu().tolist() == want[1]
    assert (kept.cpu().numpy() == want[0]).all(), np.argwhere(kept.cpu().numpy() != want[0])[:4]
    for x, y in zip([x for x in (p.dk, p.dv, p.dks, p.dvs, p.dw) if x is not None], want[2]):
        x, y = (t.view({2: torch.int16, 4: torch.int32, 1: torch.int8}[t.element_size()]) for t in (x.cpu(), y))
        assert torch.equal(x, y), (x != y).nonzero()[:4]
    assert torch.equal(p.db.cpu(), p.bounds)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("heads, dim, page", [(2, 64, 16), (3, 128, 64), (1, 80, 32), (2, 16, 128), (1, 112, 256), (2, 48, 16)])
@pytest.mark.parametrize("inplace", [True, False])
def test_rows(heads, dim, page, inplace, cache):
    lens = [1, page, 3 * page + 5, 700, 2 * page - 1]
    for keep in ([1, 7, 60, 300, page], [0, 1000, 2 * page, 699, 17]):
        p = Row(lens, heads, dim, page, cache, seed=1)
        evict(p, keep, to=None if inplace else p.fresh([-(-n // page) for n in lens]))


@pytest.mark.parametrize("first, recent", [(0, 0), (1, 0), (0, 1), (50, 0), (0, 50), (30, 30), (1 << 30, 5), (3, 1 << 30)])
def test_ends_that_stay(first, recent):
    p = Row([200, 40, 30], 2, 32, 16, seed=2)
    evict(p, [50, 50, 10], first, recent)


@pytest.mark.parametrize("n", [1025, 8191, 8193, 20000, 32768, 33000])
@pytest.mark.parametrize("inplace", [True, False])
def test_long_rows(n, inplace):
    p = Row([n, n // 3], 1, 16, 64, "s8", layers=1, seed=3)
    evict(p, [n // 2, 100], 4, 100, to=None if inplace else p.fresh([n // 128 + 1, 3]))


@pytest.mark.parametrize("inplace", [True, False])
def test_equal_and_unusual_weights(inplace):
    def tied(w):
        w.copy_((w * 2).round())

    def odd(w):
        w.view(-1)[::5], w.view(-1)[1::7], w.view(-1)[2::11], w.view(-1)[3::13] = float("nan"), float("inf"), -float("inf"), -0.0

    for change in (tied, odd, torch.Tensor.zero_, lambda w: w.fill_(float("nan"))):
        for n in (300, 9000):
            p = Row([n, 77], 2, 16, 16, seed=4, layers=1)
            evict(p, [n // 3, 40], 1, 3, to=None if inplace else p.fresh([n // 48 + 1, 3]), change=change)


def test_pages_and_lengths_that_are_not_there():
    p = Row([100, 60, 40], 2, 32, 16, seed=5, width=4)         # (a row names 64 tokens)
    evict(p, [90, 30, -3])
    p = Row([100, 60, 40], 2, 32, 16, seed=6)
    to = p.fresh([2, 1, 3])         # too few pages: what has none is lost
    to[2, 0] = 1 << 29
    evict(p, [60, 30, 20], to=to)
    evict(p, [60, 30, 20], most=25)
    p.lens = [0, -4, 40]
    evict(p, [10, 10, 10])


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_evicting_twice_and_in_a_graph(cache):
    """Rows cut down, grown and cut down again in place, by replays of one graph."""
    p = Row([300, 200], 2, 64, 16, cache, seed=7)
    c, _ = p.on_device()
    table, lens, keep = ints(p.table), ints(p.lens), ints([150, 99])
    kept = torch.empty((2, 2, 2, 150), dtype=torch.int32, device="cuda")
    out = torch.empty(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side_stream()):
        sp.spmm_cache_evict(c, table, lens, keep, sp.make_evict(3, 20, 150), table, out, kept, stream())
    for _ in range(3):
        p.dw.exponential_()
        want = p.evicted([150, 99], 3, 20, 150, p.table)
        graph.replay()
        torch.cuda.synchronize()
        assert (kept.cpu().numpy() == want[0]).all() and out.cpu().tolist() == [150, 99]
        for x, y in zip([x for x in (p.dk, p.dv, p.dks, p.dvs, p.dw) if x is not None], want[2]):
            assert torch.equal(torch.nan_to_num(x.cpu().float(), 7.0), torch.nan_to_num(y.float(), 7.0))


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("has", [(True, True), (True, False), (False, True)])
def test_pages_take_their_bounds_and_weights_along(has, cache):
    """Fork, compact and copy move all parts that the cache has."""
    p = Row([50, 33], 2, 80, 16, cache, seed=8, spare=4)
    p.on_device()
    parts = [x for x in (p.dk, p.dv, p.dks, p.dvs) if x is not None] + [x for x, is_there in zip((p.db, p.dw), has) if is_there]
    c = sp.make_cache(p.dk, p.dv, p.dks, p.dvs, p.db if has[0] else None, p.dw if has[1] else None)
    old = [p.db.clone(), p.dw.clone()]
    work, info = torch.empty(sp.spmm_cache_work_bytes(c, 4), dtype=torch.uint8, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    table, out, lens = ints(p.table), ints(np.zeros((4, p.width))), ints([0] * 4)
    want = [x.clone() for x in parts]
    sp.spmm_cache_fork(c, table, ints(p.lens), ints([0, 0, 1, 1]), ints([50, 50, 33, 33]), ints([51, 51, 34, 34]), out, lens, info, work, stream())
    for j, b, i in ((1, 0, 3), (3, 1, 2)):
        for x in want:
            x[:, out[j, i].item()] = x[:, p.table[b, i].item()]
    same = lambda: all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(parts, want))      # noqa: E731
    torch.cuda.synchronize()
    assert info.cpu().tolist()[:2] == [0, 2] and same()
    before, after = out.clone(), torch.empty_like(out)
    sp.spmm_cache_compact(c, out, after, info, work, stream())
    torch.cuda.synchronize()
    moves = {(a, b) for a, b in zip(before.flatten().tolist(), after.flatten().tolist()) if a >= 0}
    for x in want:
        y = x.clone()
        for a, b in moves:
            x[:, b] = y[:, a]
    assert same() and info[1].item() == sum(a != b for a, b in moves)
    n = p.pages
    sp.spmm_cache_copy(c, ints([0, 1]), ints([n - 1, n - 2]), 2, stream())
    torch.cuda.synchronize()
    for x in want:
        x[:, n - 1], x[:, n - 2] = x[:, 0], x[:, 1]
    assert same()
    for x, y, is_there in zip((p.db, p.dw), old, has):
        assert is_there or torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
