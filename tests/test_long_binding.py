"""The calls of long contexts as they are marshalled in C, against those in Python: the same descriptions, the same refusals, the same results."""
import pytest
import torch

import paper_2306_16601_amd as sp
from paper_2306_16601_amd import cache_binding as cb
from long_reference import Long, stream

pytestmark = pytest.mark.gpu


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def p():
    p = Long([1, 2], [70, 33], 4, 2, 64, 16, layers=2, seed=1)
    p.on_device()
    return p


def test_descriptions_are_the_same(p):
    for name, args in (("make_cache", (p.dk, p.dv, None, None, p.db, p.dw)), ("make_cache", (p.dk, p.dv, None, None, p.db)), ("make_cache", (p.dk, p.dv, None, None, None, p.dw)),
                       ("make_select", (8, 5, 1, 2, True, 9)), ("make_weigh", (8, 1 << 40, 0.25, False, 3, 0.5)), ("make_evict", (1, 2, 1 << 33))):
        assert type(getattr(sp, name)(*args)).__name__ == "spmm_cache_record"
        assert bytes(memoryview(getattr(sp, name)(*args))) == bytes(memoryview(cb._in_python[name](*args))), name
    assert bytes(memoryview(sp.make_select(8, 5))) == bytes(memoryview(sp.make_select(8, 5, 1, 1, True, 0)))


def test_what_is_wrong_is_refused_either_way(p):
    c, b = p.cache, p.batch
    how, att, wei, evi = sp.make_select(4, 5, 1, 1, True, 0), sp.make_attend(4, 2, 0.125, True, 0, "bf16"), sp.make_weigh(4, 2, 0.125, True, 0, 1.0), sp.make_evict(1, 2, 20)
    q, scores, lists, out = p.q.cuda(), torch.zeros((3, 2, p.width), device="cuda"), ints(3, 2, 5), torch.zeros((256, 3), dtype=torch.bfloat16, device="cuda")
    work = torch.zeros(sp.spmm_weigh_work_bytes(c, b, 3, wei), dtype=torch.uint8, device="cuda")
    big = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    table, lens, kept = ints(2, p.width), ints(2), ints(2, 2, 2, 20)
    calls = [
        ("make_cache", (p.dk, p.dv, None, None, p.db[:1])), ("make_cache", (p.dk, p.dv, None, None, p.db.float())), ("make_cache", (p.dk, p.dv, None, None, None, p.dw.double())),
        ("make_cache", (p.dk, p.dv, None, None, None, p.dw[..., :8].contiguous())), ("make_cache", (p.dk, p.dv, None, None, p.db.cpu())),
        ("spmm_cache_score", (c, 0, b, q[:2], 3, how, scores, p.width, None)), ("spmm_cache_score", (c, 0, b, q, 3, how, scores, p.width + 1, None)),
        ("spmm_cache_score", (c, 0, b, q, 3, how, scores.half(), p.width, None)), ("spmm_cache_select", (c, b, scores[:2], 3, p.width, how, lists, None)),
        ("spmm_cache_select", (c, b, scores, 3, p.width, how, lists[:2], None)), ("spmm_cache_select", (c, b, scores, 3, p.width, how, lists.long(), None)),
        ("spmm_cache_attend_selected", (c, 0, b, q, 3, att, lists, 6, out, 3, big, None)), ("spmm_cache_attend_selected", (c, 0, b, q, 3, att, lists, 5, out.float(), 3, big, None)),
        ("spmm_cache_attend_selected", (c, 0, b, q, 3, att, lists, 5, out, 4, big, None)), ("spmm_cache_attend_selected", (c, 0, b, q, 3, att, lists, 5, out, 3, ints(1), None)),
        ("spmm_cache_weigh", (c, 0, b, q.float(), 3, wei, work, None)), ("spmm_cache_weigh", (c, 0, b, q, 3, wei, work[:-1].clone(), None)),
        ("spmm_cache_evict", (c, table, lens, ints(3), evi, table, ints(2), kept, None)), ("spmm_cache_evict", (c, table, lens, lens, evi, ints(2, 3), ints(2), kept, None)),
        ("spmm_cache_evict", (c, table, lens, lens, evi, table, ints(2), kept[:1].clone(), None)),
    ]
    for name, args in calls:
        with pytest.raises(ValueError):
            getattr(sp, name)(*args)
        with pytest.raises(ValueError):
            cb._in_python[name](*args)
    none = sp.make_cache(p.dk, p.dv)
    for name, args in (("spmm_cache_bounds", (none, 0, b, 3)), ("spmm_cache_bounds", (c, 2, b, 3)), ("spmm_cache_score", (none, 0, b, q, 3, how, scores, p.width)),
                       ("spmm_cache_weigh", (none, 0, b, q, 3, wei, work)), ("spmm_cache_evict", (none, table, lens, lens, evi, table, ints(2), kept)),
                       ("spmm_cache_select", (c, b, scores, 3, p.width, sp.make_select(4, 5, 3, 3), lists)), ("spmm_selected_work_bytes", (c, 0, att, 5)),
                       ("spmm_weigh_work_bytes", (c, b, 3, sp.make_weigh(4, 2, 0.125, True, 0, 2.0)))):
        with pytest.raises(sp.SpmmError):
            getattr(sp, name)(*args)
        with pytest.raises(sp.SpmmError):
            cb._in_python[name](*args)


def test_either_way_computes_the_same(p):
    """Records made in C, keywords, ctypes structures and raw addresses."""
    c, b = p.cache, p.batch
    q, out = p.q.cuda(), []
    for f in ({n: getattr(sp, n) for n in cb._in_python}, cb._in_python):
        scores, lists, o = torch.zeros((3, 2, p.width), device="cuda"), ints(3, 2, 5), torch.zeros((256, 3), device="cuda")
        how, att = f["make_select"](4, 5, 1, 1, True, 0), f["make_attend"](4, 2, 0.125, True, 0, "f32")
        f["spmm_cache_bounds"](c, 0, b, 3, stream())
        f["spmm_cache_score"](c, 0, b, q, T=3, how=how, scores=scores, lds=p.width, stream=stream())
        f["spmm_cache_select"](c, b, scores.data_ptr(), 3, p.width, how, lists, stream())
        work = torch.zeros(f["spmm_selected_work_bytes"](c, 3, att, 5), dtype=torch.uint8, device="cuda")
        f["spmm_cache_attend_selected"](c, 0, b, q, 3, att, lists, 5, o, 3, work)
        p.dw.fill_(1.0)
        wei = f["make_weigh"](4, 2, 0.125, True, 0, 0.5)
        more = torch.zeros(f["spmm_weigh_work_bytes"](c, b, 3, wei), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        f["spmm_cache_weigh"](c, 0, b, q, 3, wei, more, stream())
        out.append((scores, lists, o, p.dw.clone()))
    torch.cuda.synchronize()
    for x, y in zip(*out):
        assert torch.equal(x, y)
