"""Build libcodecgauge.so in-tree with nvcc for sm_103a (one -gencode, TUs in parallel)."""
from __future__ import annotations

import importlib.util
import os
import runpy
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

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        calls = ex.submit(_build_calls, force)
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
        calls.result()
    return LIB


def _build_calls(force: bool) -> None:
    """The short way from Python to some entry points (csrc/cg_calls.cpp), for this interpreter and torch. The library does
    without it: where it cannot be built, none is left (an older one might make the calls of then), and the calls go by ctypes."""
    try:
        why = _compile_calls(force)
    except OSError as e:   # (no compiler, no torch.version, ...)
        why = str(e)
    if why:
        sys.stderr.write(f"{why}\ncalls go by ctypes\n")
        if os.path.exists(CALLS):
            os.remove(CALLS)


def _compile_calls(force: bool) -> str:
    """Why the module could not be built; empty: it is there."""
    src, inc = os.path.join(CSRC, "cg_calls.cpp"), sysconfig.get_path("include")
    spec = importlib.util.find_spec("torch")
    torch = os.path.dirname(spec.origin) if spec and spec.origin else ""
    for h in (os.path.join(inc, "Python.h"), os.path.join(torch, "include/torch/csrc/autograd/python_variable.h")):
        if not os.path.exists(h):
            return f"no {h}"
    version = runpy.run_path(os.path.join(torch, "version.py"))["__version__"]
    built_for = os.path.join(BUILD_DIR, f"calls-{version}")
    headers = [os.path.join(HERE, "..", "include", f) for f in ("codecgauge_tree.h", "codecgauge_block8.h", "codecgauge_paged.h")]
    if not (force or _stale(CALLS, [src, *headers, __file__]) or _stale(built_for, [CALLS])):
        return ""
    tmp = CALLS + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-fvisibility=hidden", f'-DCG_TORCH_VERSION="{version}"',
           f"-I{inc}", f"-I{torch}/include", f"-I{torch}/include/torch/csrc/api/include", src, f"-L{torch}/lib", "-ltorch_python",
           "-ltorch_cpu", "-lc10", "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        return f"g++ failed: {' '.join(cmd)}\n{r.stderr}"
    os.replace(tmp, CALLS)
    open(built_for, "w").close()
    return ""


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose=True, ptxas_verbose="--ptxas" in sys.argv)
    print(LIB)
