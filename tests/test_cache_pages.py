"""spmm_cache_fork, spmm_cache_compact and spmm_cache_copy on the device against their definitions, row by row.  All of it is exact."""
import numpy as np
import pytest
import torch

import paper_2306_16601_amd as sp
from cache_reference import side_stream

pytestmark = pytest.mark.gpu


def pool(layers, pages, heads, page, dim, kind, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "bf16":
        k, v = (torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((layers, pages, heads, page, dim), (layers, pages, heads, dim, page)))
        return [k, v]
    k, v = (torch.randint(-128, 128, s, generator=g, dtype=torch.int8).cuda() for s in ((layers, pages, heads, page, dim), (layers, pages, heads, dim, page)))
    ks, vs = (torch.rand((layers, pages, heads, page), generator=g).cuda() for _ in range(2))
    return [k, v, ks, vs]


def fork_by_rows(table, lens, parent, keep, want, pages, page):
    """(table, lengths, copies, missing) by the header's rules"""
    width = table.shape[1]
    valid = lambda p: 0 <= p < pages        # noqa: E731
    used = {int(p) for p in table.flatten() if valid(p)}
    free = iter(sorted(set(range(pages)) - used))
    kept = [max(0, min(k, int(lens[p]), width * page)) if 0 <= p < len(lens) else 0 for p, k in zip(parent, keep)]
    whole = {int(table[p, i]) for p, k in zip(parent, kept) if 0 <= p < len(lens) for i in range(k // page)}
    owner = {}
    for j, (p, k) in enumerate(zip(parent, kept)):
        if k % page:
            owner.setdefault(int(table[p, k // page]), j)
    out, copies, missing = np.full((len(parent), width), -1, np.int32), [], 0

    def take():
        nonlocal missing
        n = next(free, None)
        missing += n is None
        return -1 if n is None else n

    for j, (p, k, w) in enumerate(zip(parent, kept, want)):
        n = k // page
        if n:
            out[j, :n] = table[p, :n]
        if k % page:
            last = int(table[p, n])
            if valid(last) and (last in whole or owner[last] != j):
                out[j, n] = take()
                copies.append((last, int(out[j, n])))
            else:
                out[j, n] = last
        for i in range(-(-k // page), -(-max(k, w) // page)):
            out[j, i] = take()
    return out, np.array(kept, np.int32), copies, missing


def fork(table, lens, parent, keep, want, pages, page=16, kind="bf16", layers=2, heads=2, dim=16, seed=0, times=1):
    t = pool(layers, pages, heads, page, dim, kind, seed)
    cache = sp.make_cache(*t)
    ref = [x.clone() for x in t]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()      # noqa: E731
    rows = len(parent)
    out, out_len = torch.full((rows, table.shape[1]), 55, dtype=torch.int32, device="cuda"), torch.full((rows,), 66, dtype=torch.int32, device="cuda")
    info = torch.full((4,), 77, dtype=torch.int32, device="cuda")
    work = torch.full((sp.spmm_cache_work_bytes(cache, rows),), 0x5a, dtype=torch.uint8, device="cuda")
    args = [dev(a) for a in (table, lens, parent, keep, want)]
    for _ in range(times):
        sp.spmm_cache_fork(cache, *args, out, out_len, info, work, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want_table, want_len, copies, missing = fork_by_rows(table, lens, parent, keep, want, pages, page)
    info = info.cpu().tolist()
    if missing:
        assert info == [missing, 0, 0, 0]
        assert (out == 55).all() and (out_len == 66).all()
        copies = []
    else:
        assert (out.cpu().numpy() == want_table).all(), np.argwhere(out.cpu().numpy() != want_table)[:5]
        assert (out_len.cpu().numpy() == want_len).all()
        assert info == [0, len(copies), len({int(p) for p in want_table.flatten() if 0 <= p < pages}), 0]
    for x, y in zip(t, ref):
        for a, b in copies:
            y[:, b] = y[:, a]
        assert torch.equal(x, y)
    return info


def rows(lens, width, pages, page=16, seed=0):
    order = np.random.default_rng(seed).permutation(pages)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for b, n in enumerate(lens):
        held = -(-n // page)
        table[b, :held] = order[at:at + held]
        at += held
    return table


@pytest.mark.parametrize("kind", ["bf16", "s8"])
@pytest.mark.parametrize("page, dim", [(16, 16), (32, 64), (128, 80)])
def test_beams_go_on_from_some_parents(page, dim, kind):
    lens = [3 * page + 5, 3 * page + 5, 2 * page, page - 1]
    table = rows(lens, 6, 40, page)
    for parent in ([0, 0, 1, 1], [3, 3, 3, 3], [2, 2, 0, 2], [0, 1, 2, 3], [3, 2, 1, 0]):
        fork(table, lens, parent, [lens[p] for p in parent], [lens[p] + 1 for p in parent], 40, page, kind, dim=dim, times=2)


def test_trim_free_and_grow():
    lens = [50, 33, 16, 0, 100]
    table = rows(lens, 8, 30)
    fork(table, lens, [0, 1, 2, 3, 4], [17, 33, 16, 0, 96], [17, 80, 16, 40, 128], 30)
    fork(table, lens, [-1, 1, -1, 4], [9, 20, 0, 1000], [0, 20, 100, 0], 30)
    fork(table, lens, [4, 4, 4], [100, 40, 48], [0, 0, 0], 30)         # a page kept whole by one row, and ended inside by another
    fork(table, lens, [-1, -1], [0, 0], [0, 0], 30)
    fork(table, lens, [7, -5, 2], [10, 10, -3], [5, -1, 1], 30)        # parents and lengths that are not there


def test_missing_pages_leave_everything():
    lens = [50, 33]
    table = rows(lens, 12, 9)
    assert fork(table, lens, [0, 0, 1], [50, 50, 33], [51, 51, 34], 9)[0] == 0
    assert fork(table, lens, [0, 0, 1], [50, 50, 33], [51, 100, 34], 9)[0] == 2
    info = fork(table[:, :4], lens, [0, 0, 1], [50, 50, 33], [51, 50, 33], 8)
    assert info[0] == 0
    # a row cannot be wider than the table
    t = pool(1, 64, 1, 16, 16, "bf16", 0)
    cache, out, out_len = sp.make_cache(*t), torch.full((1, 4), 5, dtype=torch.int32, device="cuda"), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    info, one = torch.zeros(4, dtype=torch.int32, device="cuda"), lambda v: torch.tensor([v], dtype=torch.int32, device="cuda")      # noqa: E731
    work = torch.empty(sp.spmm_cache_work_bytes(cache, 1), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_fork(cache, torch.full((1, 4), -1, dtype=torch.int32, device="cuda"), one(0), one(-1), one(0), one(65), out, out_len, info, work, None)
    torch.cuda.synchronize()
    assert info[0] > 0 and (out == 5).all() and out_len[0] == 5


@pytest.mark.parametrize("seed", range(12))
def test_random_generations(seed):
    r = np.random.default_rng(seed)
    page, n, m = int(r.choice([16, 32, 64])), int(r.integers(1, 70)), int(r.integers(1, 70))
    lens = r.integers(0, 5 * page, n)
    table = rows(lens, 7, 1500, page, seed)
    for b in range(1, n):       # some rows share their first pages
        if r.random() < 0.4:
            i = min(int(lens[b - 1]), int(lens[b])) // page
            table[b, :i] = table[b - 1, :i]
    parent = r.integers(-1, n, m)
    keep = np.where(r.random(m) < 0.6, 10 ** 6, r.integers(0, 5 * page, m))
    fork(table, lens, parent, keep, r.integers(0, 7 * page, m), 1500, page, layers=1, heads=1, seed=seed)


def test_many_rows_and_pages():
    """More rows, and more pages, than a workgroup has threads."""
    r = np.random.default_rng(5)
    lens = r.integers(1, 60, 1500)
    table = rows(lens, 4, 9000)
    fork(table, lens, r.integers(0, 1500, 2100), np.full(2100, 64), r.integers(0, 64, 2100), 9000, layers=1, heads=1)
    fork(rows([100] * 50, 9, 70000, seed=3), [100] * 50, list(range(50)) * 2, [100] * 100, [101] * 100, 70000, layers=1, heads=1)


def compact(table, pages, kind="bf16", layers=2, heads=2, page=16, dim=16, in_place=False, seed=0):
    t = pool(layers, pages, heads, page, dim, kind, seed)
    cache = sp.make_cache(*t)
    ref = [x.clone() for x in t]
    src = torch.from_numpy(table).cuda()
    out = src if in_place else torch.full_like(src, 55)
    info = torch.full((4,), 77, dtype=torch.int32, device="cuda")
    work = torch.full((sp.spmm_cache_work_bytes(cache, table.shape[0]),), 0x5a, dtype=torch.uint8, device="cuda")
    sp.spmm_cache_compact(cache, src, out, info, work, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    used = sorted({int(p) for p in table.flatten() if 0 <= p < pages})
    moves = dict(zip([p for p in used if p >= len(used)], sorted(set(range(len(used))) - set(used))))
    assert (out.cpu().numpy() == np.vectorize(lambda p: moves.get(int(p), int(p)))(table)).all()
    assert info.cpu().tolist() == [0, len(moves), len(used), 0]
    for x, y in zip(t, ref):
        for a, b in moves.items():
            y[:, b] = y[:, a]
        assert torch.equal(x, y)


@pytest.mark.parametrize("kind", ["bf16", "s8"])
@pytest.mark.parametrize("page, dim", [(16, 16), (64, 128)])
@pytest.mark.parametrize("in_place", [True, False])
def test_compact(page, dim, in_place, kind):
    r = np.random.default_rng(page)
    for pages, used in ((40, 13), (40, 40), (40, 1), (300, 150), (1, 1)):
        table = np.full(used + 7, -1, np.int32)
        table[:used] = r.permutation(pages)[:used]
        table[used:used + 3] = table[0]         # shared
        compact(r.permutation(np.concatenate((table, [-1] * (-len(table) % 4))).astype(np.int32)).reshape(4, -1), pages, kind, page=page, dim=dim, in_place=in_place)
    compact(np.full((3, 5), -1, np.int32), 20, kind, page=page, dim=dim, in_place=in_place)
    compact(np.array([[7, 20, -3, 1 << 30]], np.int32), 20, kind, page=page, dim=dim, in_place=in_place)    # numbers outside the pool


def test_compact_a_large_pool():
    r = np.random.default_rng(1)
    compact(r.permutation(70000)[:20000].astype(np.int32).reshape(100, 200), 70000, layers=1, heads=1)


@pytest.mark.parametrize("kind", ["bf16", "s8"])
@pytest.mark.parametrize("heads, page, dim", [(1, 16, 16), (3, 32, 80), (8, 128, 128)])
def test_copy(heads, page, dim, kind):
    t = pool(3, 50, heads, page, dim, kind, 3)
    cache = sp.make_cache(*t)
    ref = [x.clone() for x in t]
    src, dst = [3, 4, 4, 9, 50, 7], [10, 11, 12, 0, 1, -1]
    for x in ref:
        for a, b in zip(src[:4], dst[:4]):
            x[:, b] = x[:, a]
    side = side_stream()
    a, b = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst))
    torch.cuda.synchronize()
    sp.spmm_cache_copy(cache, a, b, 6, side.cuda_stream)
    sp.spmm_cache_copy(cache, a, b, 0, side.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(t, ref))
