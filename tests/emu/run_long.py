"""Runs calls for long contexts through the host emulation and compares them with their definitions (tests/long_reference.py).  Called as a subprocess, which prints a line for each: an access
outside the operands ends it with a segmentation fault, a barrier that not all waves reach with the emulator's deadlock report.
usage: run_long.py JSON ...     {"call": "selected" | "weigh" | "bounds" | "score" | "evict", "problem": arguments of Long, and what the call takes}"""
import ctypes
import json
import os
import sys

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
sys.path[:0] = [ROOT, os.path.dirname(HERE), HERE]

import build_long_emu  # noqa: E402
import torch  # noqa: E402

from long_exact import compare, limits, plant, share, shared_weights  # noqa: E402
from long_reference import POISON, Long, kept_of  # noqa: E402
from paper_2306_16601_amd import cache_binding as cb  # noqa: E402

lib = ctypes.CDLL(build_long_emu.LIB)
lib.emu_alloc.restype = ctypes.c_void_p
lib.emu_alloc.argtypes = [ctypes.c_size_t]


class Device:
    """An array in memory of its own, which ends at a protected page."""

    def __init__(self, a):
        if isinstance(a, torch.Tensor):
            a = a.view(torch.int16).numpy() if a.dtype == torch.bfloat16 else a.numpy()
        a = np.ascontiguousarray(a)
        self.shape, self.dtype, self.size = a.shape, a.dtype, a.nbytes
        self.at = lib.emu_alloc(max(a.nbytes, 16))
        ctypes.memmove(self.at, a.ctypes.data, a.nbytes)

    def back(self):
        a = np.empty(self.shape, self.dtype)
        ctypes.memmove(a.ctypes.data, self.at, self.size)
        return a


def call(name, *args):
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else ctypes.c_void_p(a.at) if isinstance(a, Device) else ctypes.c_void_p() if a is None else a for a in args]
    rc = getattr(lib, name)(*args)
    assert rc == 0, (name, rc)


i64, i32 = ctypes.c_int64, ctypes.c_int32


def described(p):
    p.d = {n: None if getattr(p, n) is None else Device(getattr(p, n)) for n in ("k", "v", "k_scale", "v_scale", "bounds", "weight", "q")}
    p.d |= {"start": Device(p.start), "lens": Device(np.asarray(p.lens, np.int32)), "table": Device(p.table)}
    at = lambda n: None if p.d[n] is None else p.d[n].at        # noqa: E731
    cache = cb.spmm_cache_t(at("k"), at("v"), at("k_scale"), at("v_scale"), int(p.kind == "s8"), p.layers, p.k.shape[2], p.dim, p.page, p.pages, at("bounds"), at("weight"))
    return cache, cb.spmm_batch_t(len(p.news), at("start"), at("lens"), at("table"), p.table.shape[1])


def random_lists(p, pages, causal, window, seed):
    r = np.random.default_rng(seed)
    lists = np.full((max(1, p.tokens), p.k.shape[2], pages), -1, np.int32)
    for t, b, at in p.columns():
        lo, hi = p.pages_seen(b, at, causal, window)
        for h in range(lists.shape[1]):
            n = min(pages, max(0, hi - lo + 1))
            lists[t, h, :n] = np.sort(r.permutation(np.arange(lo, hi + 1))[:n])
    return lists


def selected(p, pages, tol=None, causal=True, window=0, scale=None, seed=0, odd=None):
    """tol: of the sum of magnitudes; without one nothing is rounded to less than binary32."""
    if odd:
        plant(p, odd)
    cache, batch = described(p)
    T, scale = max(1, p.tokens), scale or p.dim ** -0.5
    lists = random_lists(p, pages, causal, window, seed)
    how = cb.spmm_attend_t(p.q_heads, max(p.news), scale, causal, window, cb.SPMM_OUT_F32, 1.0, 0)
    n = i64()
    call("spmm_selected_work_bytes", cache, i64(T), how, i64(pages), ctypes.byref(n))
    out = Device(np.full((p.q_heads * p.dim, T), POISON, np.float32))
    call("spmm_cache_attend_selected", cache, i32(p.layer), batch, p.d["q"], i64(T), how, Device(lists), i64(pages), out, i64(T), Device(np.full(n.value, 255, np.uint8)), None)
    if odd:
        bad, *where = compare(out.back().astype(np.float64), p, lists, scale, causal, window)
        return {"bad": bad, "where": where}
    ref, mag = p.selected_wanted(lists, scale, causal=causal, window=window) if tol else limits(p, lists, scale, causal, window)
    return compared(out.back(), np.where(np.isnan(mag), POISON, ref), np.where(np.isnan(mag), 0, mag) * (tol or 1))


def weigh(p, tol, max_new=None, causal=True, window=0, decay=0.5, shared=()):
    share(p, shared)
    cache, batch = described(p)
    T = max(1, p.tokens)
    how = cb.spmm_weigh_t(p.q_heads, max_new or max(p.news), p.dim ** -0.5, causal, window, decay)
    n = i64()
    call("spmm_weigh_work_bytes", cache, batch, i64(T), how, ctypes.byref(n))
    call("spmm_cache_weigh", cache, i32(p.layer), batch, p.d["q"], i64(T), how, Device(np.full(n.value, 255, np.uint8)), None)
    want, added = (shared_weights if shared else Long.weights_wanted)(p, max_new or max(p.news), p.dim ** -0.5, causal, window, decay)
    return compared(p.d["weight"].back(), want, tol * added + 2.0 ** -22 * np.abs(want))


def bounds(p, T=None):
    cache, batch = described(p)
    want = p.bounds_wanted()
    call("spmm_cache_bounds", cache, i32(p.layer), batch, i64(T or max(1, p.tokens)), None)
    got = torch.from_numpy(p.d["bounds"].back()).view(torch.bfloat16).double()
    return compared(got.numpy(), want.numpy(), 0.0 if p.kind == "bf16" else np.abs(want.numpy()) * (2.0 ** -8 + 2.0 ** -22))


def score(p, causal=True, window=0, pad=0, pages=5, first=1, last=1):
    """And select, of what it gives."""
    cache, batch = described(p)
    T, heads, lds = max(1, p.tokens), p.k.shape[2], p.table.shape[1] + pad
    how = cb.spmm_select_t(p.q_heads, pages, first, last, causal, window)
    out, lists = Device(np.full((T, heads, lds), POISON, np.float32)), Device(np.full((T, heads, pages), POISON, np.int32))
    call("spmm_cache_score", cache, i32(p.layer), batch, p.d["q"], i64(T), how, out, i64(lds), None)
    call("spmm_cache_select", cache, batch, out, i64(T), i64(lds), how, lists, None)
    got = out.back()
    want, mag, mine = p.scores_wanted(causal, window)
    full, tol = np.full(got.shape, float(POISON)), np.zeros(got.shape)
    full[mine, :, :lds - pad], tol[:, :, :lds - pad] = want[mine], mag * 2.0 ** -23 * (2 * p.dim + 2)
    said = compared(got, full, tol)
    wrong = int((lists.back() != p.lists_wanted(got, pages, first, last, causal, window)).sum())
    return said | {"bad": said["bad"] + wrong, "lists": wrong}


def evict(p, keep, first, recent, most, inplace):
    """To the same pages, or to new ones (behind the old ones in the pool)."""
    if not inplace:
        tail = lambda x: None if x is None else torch.cat((x, x.flip(1)), 1)        # noqa: E731
        p.k, p.v, p.k_scale, p.v_scale, p.weight, p.bounds = (tail(getattr(p, n)) for n in ("k", "v", "k_scale", "v_scale", "weight", "bounds"))
    to = p.table.copy() if inplace else np.where(p.table >= 0, 2 * p.pages - 1 - p.table, -1).astype(np.int32)
    p.pages = p.k.shape[1]
    cache, batch = described(p)
    rows, heads = len(p.news), p.k.shape[2]
    kept, lens = Device(np.full((p.layers, rows, heads, most), POISON, np.int32)), Device(np.full(rows, POISON, np.int32))
    call("spmm_cache_evict", cache, p.d["table"], i64(p.table.shape[1]), p.d["lens"], i64(rows), Device(np.full(rows, keep, np.int32)), cb.spmm_evict_t(first, recent, most), Device(to), lens,
         kept, None)
    bad, kept = 0, kept.back()
    want = {n: getattr(p, n).clone() for n in ("k", "v", "weight") + (("k_scale", "v_scale") if p.kind == "s8" else ())}
    for b in range(rows):
        n = min(keep, p.held(b), most)
        bad += int(lens.back()[b] != n)
        for i in range(p.layers):
            for h in range(heads):
                j = np.arange(p.held(b))
                ids = kept_of(p.weight[i, p.table[b, j // p.page], h, j % p.page].numpy(), n, first, recent)
                bad += int((kept[i, b, h] != ids + [-1] * (most - n)).sum())
                src, dst = np.asarray(ids, int), np.arange(n)
                for name, x in want.items():
                    old = getattr(p, name)
                    if name == "v":
                        x[i, to[b, dst // p.page], h, :, dst % p.page] = old[i, p.table[b, src // p.page], h, :, src % p.page]
                    else:
                        x[i, to[b, dst // p.page], h, dst % p.page] = old[i, p.table[b, src // p.page], h, src % p.page]
    for name, x in want.items():
        got = p.d[name].back()
        same = got.view(np.uint8).reshape(-1) == Device(x).back().view(np.uint8).reshape(-1)
        bad += int((~same).sum())
    return {"bad": bad}


def compared(got, want, tol):
    got = got.astype(np.float64)
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want)))
    return {"bad": int(bad.sum()), "where": np.argwhere(bad)[:3].tolist(), "got": got[bad][:3].tolist(), "want": want[bad][:3].tolist()}


def main():
    for text in sys.argv[1:]:
        case = json.loads(text)
        p = Long(**case.pop("problem"))
        for name in ("lens", "table"):
            if name in case:
                setattr(p, name, np.asarray(case.pop(name), np.int32) if name == "table" else case.pop(name))
        print(json.dumps({"selected": selected, "weigh": weigh, "bounds": bounds, "score": score, "evict": evict}[case.pop("call")](p, **case)), flush=True)


if __name__ == "__main__":
    main()
