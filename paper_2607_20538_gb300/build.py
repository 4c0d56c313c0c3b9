"""Build libcodecgauge.so in-tree with nvcc for sm_103a (one -gencode, TUs in parallel)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcodecgauge.so")
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))   # (of this interpreter)
BUILD_DIR = os.path.join(HERE, "_build")
SOURCES = ["cg_api.cu", "cg_simt.cu", "cg_tc.cu", "cg_tc_rows.cu", "cg_tc_dec.cu", "cg_tc_keydec.cu",
           "cg_noalloc.cu", "cg_attn.cu", "cg_paged.cu", "cg_paged_attn.cu",
           "cg_paged_chunk.cu", "cg_tree.cu", "cg_block8.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    raise RuntimeError("nvcc not found")


def _flags(extra=()):
    return [*ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
            "-Xcompiler", "-fvisibility=hidden",
            "--expt-relaxed-constexpr", *extra]


def _stale(obj: str, deps: list[str]) -> bool:
    if not os.path.exists(obj):
        return True
    t = os.path.getmtime(obj)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, ptxas_verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    inc = os.path.join(HERE, "..", "include")
    headers += [os.path.join(inc, f) for f in os.listdir(inc) if f.endswith(".h")]
    extra = ["-Xptxas", "-v"] if ptxas_verbose else []
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD_DIR, src.replace(".cu", ".o"))
        if force or ptxas_verbose or _stale(o, [s, *headers, __file__]):
            jobs.append([nvcc(), *_flags(extra), "-c", s, "-o", o])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        for cmd, r in ex.map(run, jobs):
            if verbose or ptxas_verbose or r.returncode:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode:
                raise RuntimeError(f"nvcc failed: {' '.join(cmd)}")
    objs = [os.path.join(BUILD_DIR, s.replace(".cu", ".o")) for s in SOURCES]
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.check_call([nvcc(), *ARCH, "-shared", "-o", tmp, *objs, "-lcudart"])
        os.replace(tmp, LIB)
    _build_calls(force)
    return LIB


def _build_calls(force: bool) -> None:
    """The short way from Python to some entry points (csrc/cg_calls.c), for this interpreter. Where its headers are
    missing the calls go by ctypes."""
    src, inc = os.path.join(CSRC, "cg_calls.c"), sysconfig.get_path("include")
    if not os.path.exists(os.path.join(inc, "Python.h")):
        sys.stderr.write(f"no Python.h in {inc}: calls go by ctypes\n")
        return
    headers = [os.path.join(HERE, "..", "include", f) for f in ("codecgauge_tree.h", "codecgauge_block8.h", "codecgauge_paged.h")]
    if force or _stale(CALLS, [src, *headers, __file__]):
        tmp = CALLS + f".tmp{os.getpid()}"
        subprocess.check_call(["gcc", "-O2", "-Wall", "-shared", "-fPIC", f"-I{inc}", src, "-o", tmp])
        os.replace(tmp, CALLS)


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True, ptxas_verbose="--ptxas" in sys.argv)
    print(LIB)
