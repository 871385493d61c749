"""Builds tests/emu/_build.long/liblong_emu.so: the paged cache's glue and its kernels for long contexts, compiled for the host against
the emulation shim (include/hip/hip_runtime.h, include_cache/long_shim.h), with two textual changes: empty inline assembly that pins a value to a register becomes
a no-op, and kernels that are launched by address are registered with their type.  Test infrastructure only."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
CSRC = os.path.join(ROOT, "paper_2306_16601_amd", "csrc_cache")
OUT = os.path.join(HERE, "_build.long")
LIB = os.path.join(OUT, "liblong_emu.so")
CXX = os.environ.get("EMU_CXX", "/opt/rocm/llvm/bin/clang++")
SOURCES = ["cache_api.cpp", "cache_attend_lists.hip", "cache_attend_selected.hip", "cache_bounds.hip", "cache_evict.hip", "cache_score.hip", "cache_select.hip", "cache_weigh.hip"]


def available() -> bool:
    return os.path.exists(CXX)


def up_to_date() -> bool:
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", f) for f in ("spmm.h", "spmm_cache.h")] + [os.path.abspath(__file__)]
    deps += [os.path.join(HERE, f) for f in ("emu.cpp", "long_emu.cpp", "include/hip/hip_runtime.h", "include_cache/long_shim.h")]
    return os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in deps)


def for_the_host(s: str) -> str:
    s = re.sub(r'asm volatile\("" : "\+v"\(([\w\[\]]+)\)\);', r'(void)\1;', s)
    s = re.sub(r'\(const void\*\)((?:cache_\w+(?:<[^<>;]*>)?)|kernel\b)', r'emu::address(\1)', s)
    if re.search(r'\basm\b', re.sub(r'//.*', '', s)):
        raise RuntimeError("inline assembly that the emulation build does not know")
    return s


def build(force: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    # (a folder of this process: several may build at once)
    mine = os.path.join(OUT, str(os.getpid()))
    src, obj = os.path.join(mine, "src"), os.path.join(mine, "obj")
    shutil.rmtree(mine, ignore_errors=True)
    os.makedirs(src)
    os.makedirs(obj)
    for f in SOURCES + [f for f in os.listdir(CSRC) if f.endswith(".h")]:
        with open(os.path.join(CSRC, f)) as i, open(os.path.join(src, f), "w") as o:
            o.write(for_the_host(i.read()))
    flags = ["-std=c++17", "-O1", "-g", "-fPIC", "-ffp-contract=off", "-w", "-mavx2", "-mfma", "-mf16c", "-D__HIPCC__", "-include", os.path.join(HERE, "include_cache", "long_shim.h"),
             "-I", os.path.join(HERE, "include"), "-I", os.path.join(HERE, "include_cache"), "-I", HERE, "-I", os.path.join(ROOT, "include"), "-I", src, "-x", "c++"]

    def run(c):
        r = subprocess.run(c, capture_output=True, text=True)
        if r.returncode:
            raise RuntimeError("emulation build failed: %s\n%s" % (" ".join(c), r.stderr[-3000:]))

    files = [os.path.join(src, f) for f in SOURCES] + [os.path.join(HERE, "long_emu.cpp")]
    objs = [os.path.join(obj, os.path.basename(f) + ".o") for f in files]
    with ThreadPoolExecutor(max(1, min(8, os.cpu_count() or 1))) as pool:
        list(pool.map(lambda fo: run([CXX, *flags, "-c", fo[0], "-o", fo[1]]), zip(files, objs)))
    run([CXX, "-shared", "-fPIC", *objs, "-lpthread", "-o", os.path.join(mine, "lib.so")])
    os.replace(os.path.join(mine, "lib.so"), LIB)
    shutil.rmtree(mine, ignore_errors=True)
    return LIB


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    print(build(force=True))
