"""Kernels for long contexts on the CPU (tests/emu): every operand ends, and a page table begins, at memory that must not be touched, and results are compared with
their definitions."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "emu"))
import build_long_emu  # noqa: E402
from long_exact import MANY, ODD, SHARED  # noqa: E402

pytestmark = pytest.mark.skipif(not build_long_emu.available(), reason="no host clang++ for the emulation build")


@pytest.fixture(scope="module", autouse=True)
def emulated():
    return build_long_emu.build()


def case(call, news, pasts, q_heads, kv_heads, dim, page, cache, problem=(), **how):
    return {"call": call, "problem": dict(news=news, pasts=pasts, q_heads=q_heads, kv_heads=kv_heads, dim=dim, page=page, cache=cache, **dict(problem)), **how}


def run_all(cases):
    r = subprocess.run([sys.executable, os.path.join(HERE, "emu", "run_long.py"), *map(json.dumps, cases)], capture_output=True, text=True, timeout=900)
    said = [json.loads(line) for line in r.stdout.strip().splitlines()]
    assert r.returncode == 0, "emulated run failed (rc %d) at %s:\n%s" % (r.returncode, cases[len(said)], r.stderr[-3000:])
    for c, x in zip(cases, said):
        assert x["bad"] == 0, (c, x)


def run(*args, **how):
    run_all([case(*args, **how)])


# weights in bfloat16 and binary16: what test_long_attend.py holds
TOL = 2.0 ** -8 + 1e-4


@pytest.mark.parametrize("new, pages", [(70, 6), (250, 2)])
@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 112])
def test_lists_of_8_bit_caches_read_no_key_behind_the_last(dim, new, pages):
    """Lists that have four waves each, and one: some of them name the pool's last page."""
    run("selected", [new, 1], [13, 30], 4, 4, dim, 16, "s8", problem=dict(spare=0, seed=1), pages=pages, tol=TOL)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("lens", [[0, 9], [-4, 9]])
def test_weights_of_a_first_row_without_tokens(lens, cache):
    """New columns, but no token (padding): nothing in front of the page table is read.  (Rows of 1024 numbers: the table begins at a protected page.)"""
    run("weigh", [20, 5], [10, 4], 2, 1, 64, 16, cache, problem=dict(width=1024, seed=2), lens=lens, tol=3e-4)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("q_heads, kv_heads, dim, page", [(4, 4, 16, 16), (5, 1, 48, 64), (6, 2, 80, 256), (40, 2, 128, 16)])
def test_no_call_leaves_its_operands(q_heads, kv_heads, dim, page, cache):
    """Pools without a spare page, tables and lists without a spare number."""
    shape = (q_heads, kv_heads, dim, page, cache, dict(spare=0, seed=3))
    run_all([case("bounds", [1, 0, 5, 3 * page + 1], [0, 9, page - 2, page], *shape), case("score", [1, 3, 1], [40, 3 * page, 5 * page + 3], *shape, pages=3),
             case("score", [70, 3], [40, 3 * page], *shape, window=50, pad=3, pages=3), case("selected", [1, 5], [600, page], *shape, pages=4, tol=TOL),
             case("weigh", [1, 2], [600, page], *shape, tol=3e-4), case("weigh", [33, 2], [300, page], *shape, tol=3e-4, window=40)] +
            [case("evict", [1, 1, 1], [300, page, 2 * page + 3], *shape, keep=120, first=3, recent=20, most=130, inplace=inplace) for inplace in (True, False)])


# (columns, heads of queries and of keys, dims): lists with several workgroups each, with four waves each, with one
FORMS = [([1, 3], 4, 2, 64), ([2], 20, 1, 80), ([70], 4, 4, 16), ([140], 32, 2, 128), ([250], 4, 4, 48), ([250], 16, 4, 96)]


@pytest.mark.parametrize("cache", ["bf16", "s8"])
@pytest.mark.parametrize("news, q_heads, kv_heads, dim", FORMS)
def test_weights_of_values_are_not_rounded(news, q_heads, kv_heads, dim, cache):
    """Small scores of a few tokens, whose weights are all alike: a rounding of them to 16 bits is many times what binary32 is off by."""
    run("selected", news, [20] * len(news), q_heads, kv_heads, dim, 16, cache, problem=dict(seed=4), pages=2, scale=0.01)


@pytest.mark.parametrize("q_heads, kv_heads, dim, new", MANY[:6:2])
def test_odd_scales_in_lists_of_8_bit_caches(q_heads, kv_heads, dim, new):
    run_all([case("selected", [new], [60], q_heads, kv_heads, dim, 16, "s8", problem=dict(seed=6), pages=4, scale=0.02, odd=odd) for odd in ODD])


@pytest.mark.parametrize("q_heads, kv_heads, dim, page, cache", [(4, 2, 64, 16, "bf16"), (2, 2, 32, 16, "s8"), (20, 1, 80, 16, "bf16"), (8, 2, 128, 64, "s8"), (6, 3, 48, 256, "bf16")])
def test_weights_of_shared_pages(q_heads, kv_heads, dim, page, cache):
    # (as many pages of another size)
    run_all([case("weigh", news, [past * page // 16 for past in pasts], q_heads, kv_heads, dim, page, cache, problem=dict(seed=7), shared=shared, tol=3e-4,
                  window=page * 5 if dim == 32 else 0) for news, pasts, shared in SHARED])
