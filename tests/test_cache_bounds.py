"""Columns, positions and keys that a sequence of the paged cache has, whatever its numbers in device memory are: the functions
that the attention kernels take them from (csrc_cache/cache_attend.h), compiled for the host, against their definition in Python's
integers.  (No GPU needed, and none is used: with what these functions must keep out, a kernel would leave its operands.)"""
import os
import random
import subprocess

import pytest

from paper_2306_16601_amd import build as B

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")

LOWEST, HIGHEST = -(1 << 31), (1 << 31) - 1
PROGRAM = r"""
#include <cstdio>
#include "cache_attend.h"
using namespace spmm_cache;
int main()
{
    int32_t start[2], len, table = 0, token;
    AttendArgs a = {};
    a.batch.q_start = start;
    a.batch.kv_len = &len;
    a.batch.table = &table;
    a.batch.n_seqs = 1;
    while (scanf("%d %d %d %ld %d %d %d %d %d %d", start, start + 1, &len, &a.batch.ld_table, &a.pool.page_shift, &a.T, &a.max_new, &a.causal, &a.window, &token) == 10) {
        const Sequence s = sequence(a, 0);
        token = token < s.tokens ? token : s.tokens - 1;
        printf("%d %d %d %d %d\n", s.first, s.tokens, s.len, s.tokens > 0 ? s.last_seen(a, token) : -1, s.tokens > 0 ? s.first_seen(a, token) : 0);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("bounds")
    (d / "bounds.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, *B.HIPCC_FLAGS, "--offload-host-only", "-I", B.CACHE_CSRC, "-x", "hip", "-c", str(d / "bounds.hip"), "-o", str(d / "bounds.o")],
                   check=True, capture_output=True)
    subprocess.run([HIPCC, str(d / "bounds.o"), "-o", str(d / "bounds")], check=True, capture_output=True)

    def run(cases):
        said = subprocess.run([str(d / "bounds")], input="\n".join(" ".join(map(str, c)) for c in cases), check=True, capture_output=True, text=True).stdout
        return [tuple(map(int, line.split())) for line in said.splitlines()]
    return run


def columns(start, end, T, max_new):
    return 0 if start < 0 else max(0, min(end, T, start + max_new) - start)


def test_columns_lie_in_the_operands(ask):
    r = random.Random(1)
    near = (LOWEST, LOWEST + 1, LOWEST + 9, -2, -1, 0, 1, 5, 100, HIGHEST - 1, HIGHEST)
    cases = [(a, b, 7, 4, 4, T, most, 1, 0, 0) for a in near for b in near for T in (1, 9, 1 << 27) for most in (1, 6, 1 << 27)]
    cases += [(r.randint(LOWEST, HIGHEST), r.randint(LOWEST, HIGHEST), 7, 4, 4, r.randint(1, 1 << 27), r.randint(1, 1 << 27), 1, 0, 0) for _ in range(2000)]
    for c, (first, tokens, *_) in zip(cases, ask(cases)):
        start, end, T, most = c[0], c[1], c[5], c[6]
        assert max(tokens, 0) == columns(start, end, T, most), c
        assert tokens <= 0 or (0 <= first and first + tokens <= T), c


def seen(start, end, kv_len, width, shift, causal, window, token):
    """(first, last) key that a column sees."""
    n = max(0, min(kv_len, width << shift))
    at = kv_len - (end - start) + token
    if at < 0:
        return 0, -1
    return min(max(0, at - window + 1), n) if window else 0, min(at, n - 1) if causal else n - 1


def test_positions_and_windows_of_any_size(ask):
    r = random.Random(2)
    windows, lengths = (0, 1, 9, 1 << 30, HIGHEST - 1, HIGHEST), (LOWEST, LOWEST + 3, -7, 0, 2, 40, 64, 1000, 1 << 30, HIGHEST - 2, HIGHEST)
    cases = [(start, start + new, n, width, shift, 100, 100, causal, w, t) for start in (0, 3) for new in (1, 7, 60) for n in lengths
             for width, shift in ((1, 4), (4, 6), ((1 << 26) - 1, 4)) for causal in (0, 1) for w in windows for t in (0, new - 1)]
    cases += [(0, HIGHEST, n, 4, 6, 100, 100, 1, w, t) for n in lengths for w in windows for t in (0, 50)]
    for _ in range(4000):
        start, new, shift = r.randint(0, 50), r.randint(1, 50), r.randint(4, 8)
        cases.append((start, start + new, r.choice((r.randint(LOWEST, HIGHEST), r.randint(-100, 2000))), r.randint(1, (1 << 30 >> shift) - 1), shift, 100, 100,
                      r.randint(0, 1), r.choice((0, r.randint(1, HIGHEST), r.randint(1, 2000))), r.randint(0, new - 1)))
    for c, (first, tokens, length, last, begin) in zip(cases, ask(cases)):
        start, end, n, width, shift, _, _, causal, window, token = c
        assert tokens > token and length == max(0, min(n, width << shift)), c
        want = seen(start, end, n, width, shift, causal, window, token)
        assert -1 <= last < max(length, 1) and 0 <= begin <= length, (c, begin, last)
        assert ((begin, last) == want) if want[0] <= want[1] else begin > last, (c, begin, last, want)
