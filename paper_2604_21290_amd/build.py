"""Build libgraphleap.so in-tree with hipcc for gfx950, and the binding's _calls.so.

    python -m paper_2604_21290_amd.build
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libgraphleap.so")
CALLS = os.path.join(PKG, "_calls.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    "-Wall",
    # keep hipcc from emitting packed fp32 VALU ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def sources() -> list:
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")))


NOISE = "is not a recognized feature for this target"


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in res.stderr.splitlines() if NOISE not in l)
    return res.returncode, err


def build_calls(verbose: bool = True) -> str:
    """Compile the native argument marshalling (csrc/calls.cpp: host code, against the
    installed torch and Python) to _calls.so."""
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    tmp = CALLS + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(base, "include"),
           "-I", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-I", "/opt/rocm/include", "-I", sysconfig.get_paths()["include"],
           os.path.join(PKG, "csrc", "calls.cpp"), "-o", tmp,
           "-L", os.path.join(base, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print("[build]", " ".join(cmd), flush=True)
    rc, err = _run(cmd)
    if rc != 0:
        raise RuntimeError(f"{cmd[0]} failed ({rc}) on calls.cpp:\n{err}")
    os.replace(tmp, CALLS)
    return CALLS


def build_library(verbose: bool = True, jobs: int | None = None) -> str:
    """Compile each source to an object in parallel, link the library, then look at
    what became of the binding's shortcut, which the library does not use."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(ROOT, "_build")
    os.makedirs(objdir, exist_ok=True)
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    jobs = jobs or min(8, os.cpu_count() or 1)
    cmds = []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src) + ".o")
        cmds.append(([hipcc, *flags, *inc, "-c", src, "-o", obj], obj))
    if verbose:
        for c, _ in cmds:
            print("[build]", " ".join(c), flush=True)
    with cf.ThreadPoolExecutor(jobs + 1) as ex:
        calls = ex.submit(build_calls, verbose)
        results = list(ex.map(lambda c: _run(c[0]), cmds))
    for (cmd, _), (rc, err) in zip(cmds, results):
        if rc != 0:
            raise RuntimeError(f"hipcc failed ({rc}) on {cmd[-3]}:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)
    tmp = LIB + ".tmp"
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *[o for _, o in cmds], "-o", tmp]
    if verbose:
        print("[build]", " ".join(link), flush=True)
    rc, err = _run(link)
    if rc != 0:
        raise RuntimeError(f"link failed ({rc}):\n{err}")
    os.replace(tmp, LIB)
    # the library is whole without the binding's shortcut, whose failure is told last; an
    # older one, which may have been built for other signatures, does not stay beside it
    failed = calls.exception()
    if failed is not None:
        if os.path.exists(CALLS):
            os.remove(CALLS)
        raise RuntimeError(f"{LIB} is built and complete, but not the binding's shortcut {CALLS}, "
                           "without which the short calls are marshalled in Python") from failed
    return LIB


if __name__ == "__main__":
    print(build_library())
