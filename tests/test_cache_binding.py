"""The paged cache's calls as they are marshalled in C, against those in Python: the same descriptions, the same refusals."""
import pytest
import torch

import paper_2306_16601_amd as sp
from paper_2306_16601_amd import cache_binding as cb

pytestmark = pytest.mark.gpu

KINDS = {"make_cache": cb.spmm_cache_t, "make_batch": cb.spmm_batch_t, "make_append": cb.spmm_append_t, "make_attend": cb.spmm_attend_t}


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def t():
    b = torch.bfloat16
    return {"k": torch.zeros((2, 5, 4, 16, 64), dtype=b, device="cuda"), "v": torch.zeros((2, 5, 4, 64, 16), dtype=b, device="cuda"),
            "k8": torch.zeros((2, 5, 4, 16, 64), dtype=torch.int8, device="cuda"), "v8": torch.zeros((2, 5, 4, 64, 16), dtype=torch.int8, device="cuda"),
            "ks": torch.zeros((2, 5, 4, 16), device="cuda"), "vs": torch.zeros((2, 5, 4, 16), device="cuda"), "w": torch.zeros(64, device="cuda"),
            "rope": torch.zeros((9, 32, 2), device="cuda"), "q": torch.zeros((9, 8, 64), dtype=b, device="cuda"), "x": torch.zeros((16 * 64, 9), device="cuda"),
            "out": torch.zeros((512, 9), dtype=b, device="cuda"), "start": torch.tensor([0, 3, 3, 9], dtype=torch.int32, device="cuda"), "len": ints(3), "table": ints(3, 2)}


def test_descriptions_are_the_same(t):
    for name, args in (("make_cache", (t["k"], t["v"])), ("make_cache", (t["k8"], t["v8"], t["ks"], t["vs"])), ("make_batch", (t["start"], t["len"], t["table"])),
                       ("make_append", (8, "f32", 1.0, 0, t["w"], None, 1e-5, t["rope"], True)), ("make_append", (8, "u8", 0.5, 7, None, t["w"], 0.0, None, False)),
                       ("make_attend", (8, 5, 0.125, True, 3, "bf16")), ("make_attend", (8, 5, 0.125, False, 0, "u8", 0.5, 9))):
        assert type(getattr(sp, name)(*args)).__name__ == "spmm_cache_record"
        assert bytes(memoryview(getattr(sp, name)(*args))) == bytes(memoryview(cb._in_python[name](*args))), name


def test_what_is_wrong_is_refused_either_way(t):
    cache, batch, how, att = sp.make_cache(t["k"], t["v"]), sp.make_batch(t["start"], t["len"], t["table"]), sp.make_append(8, "f32", 1.0, 0, t["w"], t["w"], 1e-6, None, False), \
        sp.make_attend(8, 6, 0.125, True, 0, "bf16")
    work = torch.zeros(sp.spmm_attend_work_bytes(cache, 3, 9, att), dtype=torch.uint8, device="cuda")
    pages = torch.zeros(sp.spmm_cache_work_bytes(cache, 3), dtype=torch.uint8, device="cuda")
    f, i = torch.zeros(63, device="cuda"), ints(4)
    calls = [
        ("make_cache", (t["k"], t["k"])), ("make_cache", (t["k"].float(), t["v"].float())), ("make_cache", (t["k"].transpose(1, 2), t["v"])), ("make_cache", (t["k8"], t["v8"])),
        ("make_cache", (t["k"], t["v"], t["ks"], t["vs"])), ("make_cache", (t["k8"], t["v8"], t["ks"], t["vs"][:1])), ("make_cache", (t["k"].cpu(), t["v"])),
        ("make_batch", (t["len"], t["len"], t["table"])), ("make_batch", (t["start"].long(), t["len"], t["table"])), ("make_batch", (t["start"], t["len"], ints(2, 3).t())),
        ("make_append", (8, "f32", 1.0, 0, t["w"].double(), None, 1e-5, None, False)), ("make_append", (8, "f32", 1.0, 0, None, None, 1e-5, t["rope"][..., 0], False)),
        ("spmm_cache_append", (cache, 0, batch, t["x"], 9, 10, how, t["q"], None)), ("spmm_cache_append", (cache, 0, batch, t["x"].double(), 9, 9, how, t["q"], None)),
        ("spmm_cache_append", (cache, 0, batch, t["x"], 9, 9, how, t["q"][:8], None)),
        ("spmm_cache_append", (cache, 0, batch, t["x"], 9, 9, sp.make_append(8, "f32", 1.0, 0, f, None, 1e-6, None, False), t["q"], None)),
        ("spmm_cache_attend", (cache, 0, batch, t["q"].float(), 9, att, t["out"], 9, work, None)), ("spmm_cache_attend", (cache, 0, batch, t["q"], 9, att, t["out"][1:].clone(), 9, work, None)),
        ("spmm_cache_attend", (cache, 0, batch, t["q"], 9, att, t["out"].float(), 9, work, None)), ("spmm_cache_attend", (cache, 0, batch, t["q"], 9, att, t["out"], 9, work[:-1].clone(), None)),
        ("spmm_cache_fork", (cache, t["table"], t["len"], ints(2), ints(3), ints(3), ints(3, 2), ints(3), i, pages, None)),
        ("spmm_cache_fork", (cache, t["table"], t["len"], ints(3), ints(3), ints(3), ints(3, 4), ints(3), i, pages, None)),
        ("spmm_cache_fork", (cache, t["table"], t["len"], ints(3), ints(3), ints(3), ints(3, 2), ints(3), i, pages[:-16].clone(), None)),
        ("spmm_cache_compact", (cache, t["table"], ints(2, 2), i, pages, None)), ("spmm_cache_compact", (cache, t["table"], ints(3, 2), ints(3), pages, None)),
    ]
    for name, args in calls:
        with pytest.raises(ValueError):
            getattr(sp, name)(*args)
        with pytest.raises(ValueError):
            cb._in_python[name](*args)
    for args in ((cache, 2, batch, t["x"], 9, 9, how, t["q"], None), (cache, 0, batch, t["x"], 0, 9, how, t["q"], None)):
        with pytest.raises(sp.SpmmError):
            sp.spmm_cache_append(*args)
    with pytest.raises(sp.SpmmError):
        sp.spmm_cache_attend(cache, 0, batch, t["q"], 9, sp.make_attend(8, 6, -1.0, True, 0, "bf16"), t["out"], 9, work, None)
    with pytest.raises(sp.SpmmError):
        sp.spmm_cache_work_bytes(cache, 0)


def test_views_and_keywords_go_through(t):
    """A view whose memory covers the call, keywords, ctypes structures and raw addresses."""
    cache, batch = sp.make_cache(k=t["k"], v=t["v"]), sp.make_batch(q_start=t["start"], kv_len=t["len"], table=t["table"])
    how = sp.make_append(8, q_weight=t["w"])
    wide = torch.zeros((16 * 64, 20), device="cuda")
    q = torch.ones_like(t["q"])
    sp.spmm_cache_append(cache, 0, batch, wide[:, 3:12], T=9, ldx=20, how=how, q=q)
    sp.spmm_cache_append(cache, 0, batch, wide[:, 3:12], 9, 20, how, q, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (q == 0).all()        # (positions before their sequences: padding)
    att = sp.make_attend(8, 6, 0.125)
    work = torch.zeros(sp.spmm_attend_work_bytes(cache, 3, 9, how=att), dtype=torch.uint8, device="cuda")
    out = torch.ones((512, 12), dtype=torch.bfloat16, device="cuda")
    sp.spmm_cache_attend(cache, 0, batch, q.data_ptr(), 9, att, out[:, 2:], 12, work, stream=0)
    torch.cuda.synchronize()
    assert (out[:, 2:11] == 0).all() and (out[:, :2] == 1).all() and (out[:, 11:] == 1).all()
