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
