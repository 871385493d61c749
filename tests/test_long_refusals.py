"""Arguments that the calls of long contexts refuse, before anything is launched (no GPU needed: addresses are never followed)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2306_16601_amd as sp
from paper_2306_16601_amd import cache_binding as cb
from test_cache_refusals import ARG, BAD_CACHES, P, UNSUPPORTED, changed, refused, status

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CACHE = cb.spmm_cache_t(P, P, None, None, sp.SPMM_CACHE_BF16, 2, 4, 64, 16, 100, P, P)
BATCH = cb.spmm_batch_t(3, P, P, P, 8)
SELECT = cb.spmm_select_t(8, 5, 1, 2, 1, 0)
ATTEND = cb.spmm_attend_t(8, 5, 0.125, 1, 0, sp.SPMM_OUT_BF16, 1.0, 0)
WEIGH = cb.spmm_weigh_t(8, 5, 0.125, 1, 0, 0.5)
EVICT = cb.spmm_evict_t(1, 2, 20)
NAN, INF = float("nan"), float("inf")


def bounds(cache=CACHE, layer=0, batch=BATCH, T=9):
    return status("spmm_cache_bounds", cache, layer, batch, T, None)


def score(cache=CACHE, layer=0, batch=BATCH, q=P, T=9, how=SELECT, out=P, lds=8):
    return status("spmm_cache_score", cache, layer, batch, q, T, how, out, lds, None)


def select(cache=CACHE, batch=BATCH, scores=P, T=9, lds=8, how=SELECT, lists=P):
    return status("spmm_cache_select", cache, batch, scores, T, lds, how, lists, None)


def selected(cache=CACHE, layer=0, batch=BATCH, q=P, T=9, how=ATTEND, lists=P, pages=5, out=P, ldo=9, work=P):
    return status("spmm_cache_attend_selected", cache, layer, batch, q, T, how, lists, pages, out, ldo, work, None)


def weigh(cache=CACHE, layer=0, batch=BATCH, q=P, T=9, how=WEIGH, work=P):
    return status("spmm_cache_weigh", cache, layer, batch, q, T, how, work, None)


def evict(cache=CACHE, table=P, ld=8, lens=P, rows=3, keep=P, how=EVICT, to=P, lens_out=2 * P, kept=P):
    return status("spmm_cache_evict", cache, table, ld, lens, rows, keep, how, to, lens_out, kept, None)


CALLS = (bounds, score, select, selected, weigh, evict)


@pytest.mark.parametrize("want, change", BAD_CACHES + [(ARG, dict(bounds=P + 8)), (ARG, dict(weight=P + 4))])
def test_caches(want, change):
    c, n = changed(CACHE, **change), ctypes.c_int64()
    assert {f(cache=c) for f in CALLS} == {want}
    assert status("spmm_selected_work_bytes", c, 9, ATTEND, 5, n) == status("spmm_weigh_work_bytes", c, BATCH, 9, WEIGH, n) == want
    assert {f(cache=None) for f in CALLS} == {ARG}


def test_parts_that_a_call_needs():
    assert bounds(changed(CACHE, bounds=None)) == score(changed(CACHE, bounds=None)) == weigh(changed(CACHE, weight=None)) == evict(changed(CACHE, weight=None)) == ARG


@pytest.mark.parametrize("want, change", [
    (ARG, dict(n_seqs=0)), (ARG, dict(q_start=None)), (ARG, dict(kv_len=None)), (ARG, dict(table=None)), (ARG, dict(ld_table=0)),
    (UNSUPPORTED, dict(ld_table=1 << 26)), (UNSUPPORTED, dict(n_seqs=1 << 21)), (UNSUPPORTED, dict(n_seqs=1 << 10, ld_table=1 << 22))])
def test_batches(want, change):
    b = changed(BATCH, **change)
    assert bounds(batch=b) == score(batch=b, lds=1 << 27) == select(batch=b, lds=1 << 27) == selected(batch=b) == weigh(batch=b) == want
    assert bounds(batch=changed(BATCH, n_seqs=65536)) == weigh(batch=changed(BATCH, n_seqs=65536)) == evict(rows=65536) == UNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(q_heads=0), dict(q_heads=6), dict(pages=0), dict(first=-1), dict(last=-1), dict(first=4), dict(first=(1 << 31) - 1, last=(1 << 31) - 1), dict(window=-1)])
def test_select(change):
    assert score(how=changed(SELECT, **change)) == select(how=changed(SELECT, **change)) == ARG


def test_select_operands():
    assert score(layer=-1) == score(layer=2) == score(q=None) == score(q=P + 8) == score(T=0) == score(how=None) == score(out=None) == score(out=P + 2) == score(lds=7) == ARG
    assert select(scores=None) == select(scores=P + 1) == select(T=0) == select(lds=7) == select(how=None) == select(lists=None) == select(lists=P + 2) == ARG
    assert bounds(layer=-1) == bounds(layer=2) == bounds(T=0) == bounds(T=-5) == ARG
    for f in (score, select):
        assert f(lds=(1 << 30) + 1) == f(how=changed(SELECT, q_heads=1 << 15)) == f(T=1 << 40) == f(how=changed(SELECT, pages=(1 << 20) + 1)) == UNSUPPORTED
        assert f(T=(1 << 20) + 1, how=changed(SELECT, q_heads=4)) == UNSUPPORTED


@pytest.mark.parametrize("want, change", [
    (ARG, dict(q_heads=0)), (ARG, dict(q_heads=6)), (ARG, dict(max_new=0)), (ARG, dict(scale=0.0)), (ARG, dict(scale=-1.0)), (ARG, dict(scale=INF)),
    (ARG, dict(scale=NAN)), (ARG, dict(window=-1)), (ARG, dict(out_type=0)), (ARG, dict(out_type=9)), (ARG, dict(out_type=sp.SPMM_OUT_U8, out_scale=0.0)),
    (ARG, dict(out_type=sp.SPMM_OUT_U8, out_zero_point=256)), (ARG, dict(out_type=sp.SPMM_OUT_S8, out_zero_point=-129)), (UNSUPPORTED, dict(q_heads=1 << 15))])
def test_attend(want, change):
    assert selected(how=changed(ATTEND, **change)) == want


def test_attend_operands():
    assert selected(layer=-1) == selected(layer=2) == selected(q=None) == selected(q=P + 8) == selected(T=0) == selected(how=None) == selected(lists=None) == ARG
    assert selected(lists=P + 1) == selected(pages=0) == selected(out=None) == selected(out=P + 1) == selected(ldo=8) == selected(work=None) == selected(work=P + 4) == ARG
    assert selected(T=1 << 40, ldo=1 << 40) == selected(ldo=1 << 41) == selected(pages=(1 << 20) + 1) == selected(T=(1 << 20) + 1, ldo=1 << 21, how=changed(ATTEND, q_heads=4)) == UNSUPPORTED
    n = ctypes.c_int64()
    f = lambda *a: status("spmm_selected_work_bytes", *a)       # noqa: E731
    assert f(CACHE, 0, ATTEND, 5, n) == f(CACHE, 9, None, 5, n) == f(CACHE, 9, ATTEND, 0, n) == f(CACHE, 9, ATTEND, 5, None) == ARG
    assert f(CACHE, 9, ATTEND, 1 << 21, n) == UNSUPPORTED
    assert f(CACHE, 9, ATTEND, 5, n) == sp.SPMM_OK and n.value > 0
    # lists in more parts than a grid has workgroups: 2^24, and 512 columns of 4 heads have 8 tiles each, in 1024 parts
    wide = changed(ATTEND, q_heads=512)
    assert f(CACHE, 1 << 18, wide, 1 << 20, n) == selected(T=1 << 18, ldo=1 << 18, how=wide, pages=1 << 20) == UNSUPPORTED
    assert f(CACHE, 512, wide, 1 << 20, n) == UNSUPPORTED and f(CACHE, 511, wide, 1 << 20, n) == sp.SPMM_OK


@pytest.mark.parametrize("want, change", [
    (ARG, dict(q_heads=0)), (ARG, dict(q_heads=6)), (ARG, dict(max_new=0)), (ARG, dict(scale=0.0)), (ARG, dict(scale=INF)), (ARG, dict(scale=NAN)), (ARG, dict(window=-1)),
    (ARG, dict(decay=-0.5)), (ARG, dict(decay=1.5)), (ARG, dict(decay=NAN)), (UNSUPPORTED, dict(q_heads=1 << 15))])
def test_weigh(want, change):
    n = ctypes.c_int64()
    assert weigh(how=changed(WEIGH, **change)) == status("spmm_weigh_work_bytes", CACHE, BATCH, 9, changed(WEIGH, **change), n) == want


def test_weigh_operands():
    assert weigh(layer=-1) == weigh(layer=2) == weigh(q=None) == weigh(q=P + 8) == weigh(T=0) == weigh(how=None) == weigh(work=None) == weigh(work=P + 4) == ARG
    assert weigh(T=1 << 40) == UNSUPPORTED
    n = ctypes.c_int64()
    f = lambda *a: status("spmm_weigh_work_bytes", *a)       # noqa: E731
    assert f(CACHE, None, 9, WEIGH, n) == f(CACHE, BATCH, 0, WEIGH, n) == f(CACHE, BATCH, 9, None, n) == f(CACHE, BATCH, 9, WEIGH, None) == ARG
    assert f(CACHE, changed(BATCH, n_seqs=65536), 9, WEIGH, n) == UNSUPPORTED
    assert f(CACHE, BATCH, 9, WEIGH, n) == sp.SPMM_OK and n.value > 0


def test_evict_operands():
    for name in ("table", "lens", "keep", "how", "to", "lens_out", "kept"):
        assert evict(**{name: None}) == ARG
    assert evict(lens_out=P) == evict(ld=0) == evict(rows=0) == ARG
    for change in (dict(first=-1), dict(recent=-1), dict(most=0)):
        assert evict(how=changed(EVICT, **change)) == ARG
    assert evict(ld=1 << 26) == evict(how=changed(EVICT, most=(1 << 30) + 1)) == evict(cache=changed(CACHE, n_layers=1 << 19)) == UNSUPPORTED
    assert evict(rows=60000, how=changed(EVICT, most=1 << 30)) == UNSUPPORTED


def test_the_binding_checks_tensors():
    """(Tensors of the host: what is right but for that is refused for that.)"""
    k, v = torch.zeros((2, 5, 4, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 5, 4, 64, 16), dtype=torch.bfloat16)
    b, w = torch.zeros((2, 5, 4, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 5, 4, 16))
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)     # noqa: E731
    refused(lambda: sp.make_cache(k, v, None, None, b, w), device=True)
    for what, bad, kind, shape in (("bounds", b[:, :4].contiguous(), "bfloat16", b.shape), ("bounds", b.float(), "bfloat16", b.shape), ("weight", w[..., :8].contiguous(), "float32", w.shape),
                                   ("weight", w.double(), "float32", w.shape), ("weight", w.transpose(1, 2), "float32", (2, 4, 5, 16))):
        refused(lambda: cb._tensor(bad, what, kind, shape))
    q, scores, lists = torch.zeros((9, 8, 64), dtype=torch.bfloat16), torch.zeros((9, 4, 8)), ints(9, 4, 5)
    out, work = torch.zeros((512, 9), dtype=torch.bfloat16), torch.zeros(sp.spmm_weigh_work_bytes(CACHE, BATCH, 9, WEIGH), dtype=torch.uint8)
    refused(lambda: sp.spmm_cache_score(CACHE, 0, BATCH, q, 9, SELECT, P, 8), device=True)
    refused(lambda: sp.spmm_cache_select(CACHE, BATCH, scores, 9, 8, SELECT, P), device=True)
    refused(lambda: sp.spmm_cache_attend_selected(CACHE, 0, BATCH, P, 9, ATTEND, lists, 5, P, 9, P), device=True)
    refused(lambda: sp.spmm_cache_weigh(CACHE, 0, BATCH, P, 9, WEIGH, work), device=True)
    refused(lambda: sp.spmm_cache_evict(CACHE, ints(3, 8), P, P, EVICT, P, P, P), device=True)
    for bad in (lambda: sp.spmm_cache_score(CACHE, 0, BATCH, q[:8], 9, SELECT, P, 8), lambda: sp.spmm_cache_score(CACHE, 0, BATCH, q.float(), 9, SELECT, P, 8),
                lambda: sp.spmm_cache_score(CACHE, 0, BATCH, P, 9, SELECT, scores, 9), lambda: sp.spmm_cache_score(CACHE, 0, BATCH, P, 9, SELECT, scores.double(), 8),
                lambda: sp.spmm_cache_select(CACHE, BATCH, scores[:8], 9, 8, SELECT, P), lambda: sp.spmm_cache_select(CACHE, BATCH, P, 9, 8, SELECT, lists.long()),
                lambda: sp.spmm_cache_select(CACHE, BATCH, P, 9, 8, SELECT, lists[:, :3].contiguous()), lambda: sp.spmm_cache_select(CACHE, BATCH, P, 9, 8, SELECT, ints(4, 9, 5).transpose(0, 1)),
                lambda: sp.spmm_cache_attend_selected(CACHE, 0, BATCH, q[:8], 9, ATTEND, P, 5, P, 9, P), lambda: sp.spmm_cache_attend_selected(CACHE, 0, BATCH, P, 9, ATTEND, lists, 6, P, 9, P),
                lambda: sp.spmm_cache_attend_selected(CACHE, 0, BATCH, P, 9, ATTEND, P, 5, out.float(), 9, P), lambda: sp.spmm_cache_attend_selected(CACHE, 0, BATCH, P, 9, ATTEND, P, 5, out, 10, P),
                lambda: sp.spmm_cache_attend_selected(CACHE, 0, BATCH, P, 9, ATTEND, P, 5, P, 9, ints(1)),
                lambda: sp.spmm_cache_weigh(CACHE, 0, BATCH, q[:8], 9, WEIGH, P), lambda: sp.spmm_cache_weigh(CACHE, 0, BATCH, P, 9, WEIGH, work[:-16].clone()),
                lambda: sp.spmm_cache_evict(CACHE, ints(3, 8).long(), P, P, EVICT, P, P, P)):
        refused(bad)
    table, lens, kept = ints(3, 8), ints(3), ints(2, 3, 4, 20)
    for args in ((table, ints(2), lens, EVICT, table, lens, kept), (table, lens, ints(4), EVICT, table, lens, kept), (table, lens, lens, EVICT, ints(3, 7), lens, kept),
                 (table, lens, lens, EVICT, table, lens.long(), kept), (table, lens, lens, EVICT, table, lens, kept[:1])):
        refused_or_device(lambda: sp.spmm_cache_evict(CACHE, *args))
    with pytest.raises(sp.SpmmError):
        sp.spmm_cache_bounds(CACHE, 2, BATCH, 9)


def refused_or_device(call):
    with pytest.raises(ValueError):
        call()


def test_structures_are_those_of_the_header(tmp_path):
    (tmp_path / "s.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "spmm_cache.h"\nint main(void) { printf("%zu %zu %zu %zu %zu", sizeof(spmm_select_t), '
                                  'sizeof(spmm_weigh_t), sizeof(spmm_evict_t), offsetof(spmm_cache_t, bounds), offsetof(spmm_cache_t, weight)); return 0; }\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    said = subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in said.split()] == [ctypes.sizeof(t) for t in (cb.spmm_select_t, cb.spmm_weigh_t, cb.spmm_evict_t)] + [cb.spmm_cache_t.bounds.offset, cb.spmm_cache_t.weight.offset]
