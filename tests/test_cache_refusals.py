"""Arguments that the paged cache's calls refuse, before anything is launched (no GPU needed: addresses are never followed)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2306_16601_amd as sp
from paper_2306_16601_amd import cache_binding as cb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, UNSUPPORTED = sp.SPMM_E_ARG, sp.SPMM_E_UNSUPPORTED
P = 1 << 20         # a 16-byte aligned address that nothing reads


def changed(struct, **kw):
    new = type(struct).from_buffer_copy(struct)
    for k, v in kw.items():
        setattr(new, k, v)
    return new


CACHE = cb.spmm_cache_t(P, P, None, None, sp.SPMM_CACHE_BF16, 2, 4, 64, 16, 100)
CACHE8 = changed(CACHE, type=sp.SPMM_CACHE_S8, k_scale=P, v_scale=P)
BATCH = cb.spmm_batch_t(3, P, P, P, 8)
APPEND = cb.spmm_append_t(8, sp.SPMM_OUT_F32, 1.0, 0, None, None, 1e-6, P, 10, 64, 0, None)
ATTEND = cb.spmm_attend_t(8, 5, 0.125, 1, 0, sp.SPMM_OUT_BF16, 1.0, 0)


def status(name, *args):
    return getattr(cb._functions(), name)(*args)


BAD_CACHES = [
    (ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(k=P + 8)), (ARG, dict(v=P + 2)), (ARG, dict(type=7)), (ARG, dict(n_layers=0)),
    (ARG, dict(n_heads=0)), (ARG, dict(head_dim=0)), (ARG, dict(page_tokens=0)), (ARG, dict(n_pages=0)), (ARG, dict(type=sp.SPMM_CACHE_S8)),
    (UNSUPPORTED, dict(head_dim=144)), (UNSUPPORTED, dict(head_dim=72)), (UNSUPPORTED, dict(page_tokens=8)), (UNSUPPORTED, dict(page_tokens=48)),
    (UNSUPPORTED, dict(page_tokens=512)), (UNSUPPORTED, dict(n_pages=1 << 31)),
]


@pytest.mark.parametrize("want, change", BAD_CACHES)
def test_caches(want, change):
    c, n = changed(CACHE, **change), ctypes.c_int64()
    assert status("spmm_cache_append", c, 0, BATCH, P, 9, 9, APPEND, P, None) == want
    assert status("spmm_cache_attend", c, 0, BATCH, P, 9, ATTEND, P, 9, P, None) == want
    assert status("spmm_cache_fork", c, P, 8, P, 3, P, P, P, 3, 2 * P, 2 * P, P, P, None) == want
    assert status("spmm_cache_compact", c, P, 8, 3, P, P, P, None) == want
    assert status("spmm_cache_copy", c, P, P, 3, None) == want
    assert status("spmm_cache_work_bytes", c, 3, n) == want
    assert status("spmm_attend_work_bytes", c, 3, 9, ATTEND, n) == want


@pytest.mark.parametrize("want, change", [
    (ARG, dict(n_seqs=0)), (ARG, dict(q_start=None)), (ARG, dict(kv_len=None)), (ARG, dict(table=None)), (ARG, dict(ld_table=0)),
    (UNSUPPORTED, dict(ld_table=1 << 26)), (UNSUPPORTED, dict(n_seqs=1 << 21)), (UNSUPPORTED, dict(n_seqs=1 << 10, ld_table=1 << 22))])
def test_batches(want, change):
    b = changed(BATCH, **change)
    assert status("spmm_cache_append", CACHE, 0, b, P, 9, 9, APPEND, P, None) == want
    assert status("spmm_cache_attend", CACHE, 0, b, P, 9, ATTEND, P, 9, P, None) == want


@pytest.mark.parametrize("want, change", [
    (ARG, dict(q_heads=0)), (ARG, dict(q_heads=6)), (ARG, dict(x_type=sp.SPMM_OUT_S32)), (ARG, dict(x_type=sp.SPMM_OUT_BF16)),
    (ARG, dict(x_type=sp.SPMM_OUT_S8, x_scale=0.0)), (ARG, dict(x_type=sp.SPMM_OUT_S8, x_scale=float("nan"))),
    (ARG, dict(x_type=sp.SPMM_OUT_S8, x_zero_point=128)), (ARG, dict(x_type=sp.SPMM_OUT_U8, x_zero_point=-1)), (ARG, dict(eps=-1.0)),
    (ARG, dict(eps=float("nan"))), (ARG, dict(rope_dim=0)), (ARG, dict(rope_dim=7)), (ARG, dict(rope_dim=66)), (ARG, dict(rope_len=0)),
    (UNSUPPORTED, dict(q_heads=1 << 15))])
def test_append(want, change):
    assert status("spmm_cache_append", CACHE, 0, BATCH, P, 9, 9, changed(APPEND, **change), P, None) == want


def test_append_operands():
    f = lambda layer=0, x=P, T=9, ldx=9, how=APPEND, q=P: status("spmm_cache_append", CACHE, layer, BATCH, x, T, ldx, how, q, None)     # noqa: E731
    assert f(layer=-1) == f(layer=2) == f(x=None) == f(T=0) == f(ldx=8) == f(how=None) == f(q=None) == f(q=P + 8) == ARG
    assert f(T=1 << 40, ldx=1 << 40) == f(ldx=1 << 41) == UNSUPPORTED


@pytest.mark.parametrize("want, change", [
    (ARG, dict(q_heads=0)), (ARG, dict(q_heads=6)), (ARG, dict(max_new=0)), (ARG, dict(scale=0.0)), (ARG, dict(scale=-1.0)), (ARG, dict(scale=float("inf"))),
    (ARG, dict(scale=float("nan"))), (ARG, dict(window=-1)), (ARG, dict(out_type=0)), (ARG, dict(out_type=9)), (ARG, dict(out_type=sp.SPMM_OUT_U8, out_scale=0.0)),
    (ARG, dict(out_type=sp.SPMM_OUT_U8, out_zero_point=256)), (ARG, dict(out_type=sp.SPMM_OUT_S8, out_zero_point=-129)), (UNSUPPORTED, dict(q_heads=1 << 15))])
def test_attend(want, change):
    assert status("spmm_cache_attend", CACHE, 0, BATCH, P, 9, changed(ATTEND, **change), P, 9, P, None) == want


def test_attend_operands():
    f = lambda layer=0, q=P, T=9, how=ATTEND, out=P, ldo=9, work=P: status("spmm_cache_attend", CACHE, layer, BATCH, q, T, how, out, ldo, work, None)   # noqa: E731
    assert f(layer=-1) == f(layer=2) == f(q=None) == f(q=P + 8) == f(T=0) == f(how=None) == f(out=None) == f(out=P + 1) == f(ldo=8) == ARG
    assert f(work=None) == f(work=P + 4) == ARG
    assert f(T=1 << 40, ldo=1 << 40) == f(ldo=1 << 41) == UNSUPPORTED
    n = ctypes.c_int64()
    assert status("spmm_attend_work_bytes", CACHE, 0, 9, ATTEND, n) == status("spmm_attend_work_bytes", CACHE, 3, 0, ATTEND, n) == ARG
    assert status("spmm_attend_work_bytes", CACHE, 3, 9, ATTEND, None) == status("spmm_attend_work_bytes", CACHE, 3, 9, None, n) == ARG
    assert status("spmm_attend_work_bytes", CACHE, 3, 9, ATTEND, n) == sp.SPMM_OK and n.value > 0


def test_pages_operands():
    def fork(**kw):
        a = dict(table=P, ld=8, lens=P, rows_in=3, parent=P, keep=P, want=P, rows=3, out=2 * P, out_len=2 * P, info=P, work=P) | kw
        return status("spmm_cache_fork", CACHE, *a.values(), None)
    for n in ("table", "lens", "parent", "keep", "want", "out", "out_len", "info", "work"):
        assert fork(**{n: None}) == ARG
    assert fork(out=P) == fork(out_len=P) == fork(work=P + 4) == fork(ld=0) == fork(rows=0) == fork(rows_in=0) == ARG
    assert fork(ld=1 << 26) == fork(rows=1 << 21) == fork(rows_in=1 << 21) == UNSUPPORTED
    for args in ((None, 8, 3, P, P, P), (P, 0, 3, P, P, P), (P, 8, 0, P, P, P), (P, 8, 3, None, P, P), (P, 8, 3, P, None, P), (P, 8, 3, P, P, None), (P, 8, 3, P, P, P + 4)):
        assert status("spmm_cache_compact", CACHE, *args, None) == ARG
    assert status("spmm_cache_copy", CACHE, P, P, -1, None) == status("spmm_cache_copy", CACHE, None, P, 1, None) == ARG
    assert status("spmm_cache_copy", CACHE, P, P, 1 << 31, None) == UNSUPPORTED
    assert status("spmm_cache_copy", CACHE, None, None, 0, None) == sp.SPMM_OK
    n = ctypes.c_int64()
    assert status("spmm_cache_work_bytes", CACHE, 0, n) == status("spmm_cache_work_bytes", CACHE, 3, None) == ARG
    assert status("spmm_cache_work_bytes", CACHE, 1 << 21, n) == UNSUPPORTED


def refused(call, device=False):
    with pytest.raises(ValueError) as e:
        call()
    assert ("on the device" in str(e.value)) == device, str(e.value)


def test_the_binding_checks_tensors():
    """(Tensors of the host: what is right but for that is refused for that.)"""
    k, v = torch.zeros((2, 5, 4, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 5, 4, 64, 16), dtype=torch.bfloat16)
    scale = torch.zeros(2, 5, 4, 16)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)     # noqa: E731
    refused(lambda: sp.make_cache(k, v), device=True)
    for bad in (lambda: sp.make_cache(k.float(), v.float()), lambda: sp.make_cache(k.transpose(1, 2), v),
                lambda: sp.make_cache(k.to(torch.int8), v.to(torch.int8)), lambda: sp.make_cache(k, v, scale, scale)):
        refused(bad)
    refused(lambda: cb._tensor(k, "v", "bfloat16", v.shape))
    refused(lambda: sp.make_batch(ints(4), ints(3), ints(3, 2)), device=True)
    for bad in (lambda: sp.make_batch(ints(3), ints(3), ints(3, 2)), lambda: sp.make_batch(ints(4).long(), ints(3), ints(3, 2))):
        refused(bad)
    refused(lambda: sp.make_append(8, rope=torch.zeros(4, 32, 2)), device=True)
    for bad in (lambda: sp.make_append(8, rope=torch.zeros(4, 32, 3)), lambda: sp.make_append(8, rope=torch.zeros(4, 32, 2).double()),
                lambda: sp.make_append(8, positions=torch.zeros(4))):
        refused(bad)

    q, x, att = torch.zeros((9, 8, 64), dtype=torch.bfloat16), torch.zeros((16 * 64, 9)), sp.make_attend(8, 5, 0.1)
    how = sp.make_append(8)
    out, work = torch.zeros((512, 9), dtype=torch.bfloat16), torch.zeros(sp.spmm_attend_work_bytes(CACHE, 3, 9, att), dtype=torch.uint8)
    refused(lambda: sp.spmm_cache_append(CACHE, 0, BATCH, x, 9, 9, how, P), device=True)
    refused(lambda: sp.spmm_cache_append(CACHE, 0, BATCH, P, 9, 9, how, q), device=True)
    refused(lambda: sp.spmm_cache_attend(CACHE, 0, BATCH, P, 9, att, out, 9, P), device=True)
    refused(lambda: sp.spmm_cache_attend(CACHE, 0, BATCH, P, 9, att, P, 9, work), device=True)
    weights, places = changed(APPEND), changed(APPEND)
    weights._keepalive = (torch.zeros(63), None, None, None)
    places._keepalive = (None, None, None, ints(8))
    for bad in (lambda: sp.spmm_cache_append(CACHE, 0, BATCH, x[:-1].clone(), 9, 9, how, P), lambda: sp.spmm_cache_append(CACHE, 0, BATCH, x, 9, 10, how, P),
                lambda: sp.spmm_cache_append(CACHE, 0, BATCH, x.double(), 9, 9, how, P), lambda: sp.spmm_cache_append(CACHE, 0, BATCH, P, 9, 9, how, q[:8]),
                lambda: sp.spmm_cache_append(CACHE, 0, BATCH, P, 9, 9, how, q.float()), lambda: sp.spmm_cache_append(CACHE, 0, BATCH, P, 9, 9, weights, P),
                lambda: sp.spmm_cache_append(CACHE, 0, BATCH, P, 9, 9, places, P),
                lambda: sp.spmm_cache_attend(CACHE, 0, BATCH, P, 9, att, out[:-1].clone(), 9, P), lambda: sp.spmm_cache_attend(CACHE, 0, BATCH, P, 9, att, out.float(), 9, P),
                lambda: sp.spmm_cache_attend(CACHE, 0, BATCH, P, 9, att, P, 9, work[:-16].clone()), lambda: sp.spmm_cache_attend(CACHE, 0, BATCH, q[:8], 9, att, P, 9, P),
                lambda: sp.spmm_cache_copy(CACHE, ints(3).long(), P, 3), lambda: sp.spmm_cache_copy(CACHE, P, ints(2), 3)):
        refused(bad)
    with pytest.raises(sp.SpmmError):
        sp.spmm_cache_append(CACHE, 2, BATCH, P, 9, 9, how, P)


def test_the_binding_declares_what_the_header_does():
    header = open(os.path.join(ROOT, "include", "spmm_cache.h")).read()
    declared = set(re.findall(r"^spmm_status_t (spmm_\w+)\(", header, flags=re.M))
    assert declared == set(sp.CACHE_EXPORTS)
    sizes = '#include <stdio.h>\n#include "spmm_cache.h"\nint main(void) { printf("%zu %zu %zu %zu", sizeof(spmm_cache_t), sizeof(spmm_batch_t), ' \
            'sizeof(spmm_append_t), sizeof(spmm_attend_t)); return 0; }\n'
    import subprocess
    import tempfile
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "s.c"), "w") as f:
            f.write(sizes)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")], check=True)
        said = subprocess.run([os.path.join(d, "s")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in said.split()] == [ctypes.sizeof(t) for t in (cb.spmm_cache_t, cb.spmm_batch_t, cb.spmm_append_t, cb.spmm_attend_t)]
