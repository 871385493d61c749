"""What the compiler made of the paged cache's kernels: vector registers that are kept in memory, and LDS, read from the metadata of the
built library.

Attention over 8-bit caches with heads of 65 to 128 dims, or two tiles of columns of 64, fills the 256 registers that a wave has
where two share a SIMD, and some that are used once a head are spilled: in the kernel for few columns before and after its loop over keys,
in the one for many columns addresses of the queries and results.  No other kernel spills any."""
import re

import pytest

pytest.importorskip("msgpack")

import paper_2306_16601_amd as sp  # noqa: E402
from test_kernel_resources import _code_objects, _kernels  # noqa: E402


@pytest.fixture(scope="module")
def kernels():
    sp.lib()
    return [k for elf in _code_objects(sp.binding.LIB_PATH) for k in _kernels(elf) if "10spmm_cache" in k[".name"]]


def most_spilled(name):
    eight = re.search(r"cache_attend_(few|many)ILi(\d+)EL17spmm_cache_type_t1E(.*)", name)
    if eight is None:
        return 0
    kernel, dim, rest = eight.groups()
    if kernel == "many":
        return 5 if dim == "128" else 0
    whole = rest.split("EEv")[0].endswith("Lb1")
    two = "Li2E" in rest
    return 0 if whole or (dim == "64") != two else 28


def test_spilled_registers(kernels):
    assert len(kernels) > 60
    over = {k[".name"]: k[".vgpr_spill_count"] for k in kernels if k[".vgpr_spill_count"] > most_spilled(k[".name"])}
    assert not over, over
    scratch = {k[".name"]: k[".private_segment_fixed_size"] for k in kernels if k[".private_segment_fixed_size"] > 4 * most_spilled(k[".name"]) + 8 * (most_spilled(k[".name"]) > 0)}
    assert not scratch, scratch


def test_workgroups_that_share_a_cu(kernels):
    """LDS for as many workgroups as a CU is meant to run: two of attention's (one where their registers fill it), of 160 KB."""
    for k in kernels:
        if "cache_attend" in k[".name"]:
            assert 2 * k[".group_segment_fixed_size"] <= 160 << 10, k[".name"]
            assert k[".vgpr_count"] <= (512 if "few" in k[".name"] else 256), k[".name"]
