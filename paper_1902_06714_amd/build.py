"""Build the HIP library (libnf.so) for gfx950 in-tree with hipcc.

    python -m paper_1902_06714_amd.build

Always recompiles; the library lands next to this file.

One process must hold one HIP runtime.  PyTorch's ROCm wheel carries its own
copy of the runtime (soname libamdhip64.so.7, the same as ROCm's), which its
libraries request by the unversioned file name.  A process that loads torch
first therefore satisfies this library's libamdhip64.so.7 with torch's copy;
loading this library first would pull in ROCm's copy and torch would then add
a second one.  The Python binding imports torch before loading the library.
"""

from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libnf.so")
SOURCES = ["nf_api.hip", "nf_kernels.hip", "nf_narrow.hip", "nf_narrow64.hip", "nf_medium.hip",
           "nf_eval.hip", "nf_calib.hip", "nf_skinny.hip",
           "nf_wide256.hip", "nf_wide128.hip", "nf_wide64.hip",
           "nf_params.hip"]
# the operators on the caller's own arrays, apart from the net's kernels
OPS = os.path.join(HERE, "csrc_ops")
OPS_SOURCES = ["nf_logprobs.hip", "nf_orth.hip", "nf_linear_i8.hip"]
# their calls with torch tensors, a Python module of host code
BIND = os.path.join(HERE, "_nfbind.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-Wall",
    # no packed fp32 instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build the library)")


def cxx():
    """A host C++ compiler; None where there is none."""
    for cand in (os.environ.get("CXX"), "g++", "c++", "/opt/rocm/llvm/bin/clang++"):
        if cand and shutil.which(cand):
            return shutil.which(cand)
    return None


def bind_commands(obj: str, out: str):
    """How the binding of the operators with tensors is compiled and linked; or, as a
    text, what it lacks here.  The library and its nets need none of it."""
    try:
        import torch
    except Exception as e:
        return f"torch cannot be imported ({e})"
    include = sysconfig.get_paths()["include"]
    if cxx() is None:
        return "there is no host C++ compiler"
    if not os.path.exists(os.path.join(include, "Python.h")):
        return f"Python's headers are not in {include}"
    home = os.path.dirname(torch.__file__)
    compile_ = [cxx(), "-O2", "-std=c++17", "-fPIC", "-Wall",
                f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                "-I", include, "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(home, "include"),
                "-isystem", os.path.join(home, "include", "torch", "csrc", "api", "include"),
                "-c", os.path.join(OPS, "nf_bind.cpp"), "-o", obj]
    link = [cxx(), "-shared", "-fPIC", obj, "-o", out, "-L", os.path.dirname(LIB), "-l:" + os.path.basename(LIB),
            "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN",
            "-Wl,-rpath," + os.path.join(home, "lib")]
    return compile_, link


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"build step failed ({res.returncode}): {' '.join(cmd)}\n"
                           f"{res.stdout}\n{res.stderr}")


def build(verbose: bool = False) -> str:
    objdir = os.path.join(ROOT, "_build")
    os.makedirs(objdir, exist_ok=True)
    paths = [os.path.join(CSRC, s) for s in SOURCES] + [os.path.join(OPS, s) for s in OPS_SOURCES]
    objs = [os.path.join(objdir, os.path.splitext(os.path.basename(p))[0] + ".o") for p in paths]
    cmds = [[hipcc(), *HIPCC_FLAGS, "-c", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", OPS,
             path, "-o", obj] for path, obj in zip(paths, objs)]
    tmp_bind = BIND + ".tmp"
    bind = bind_commands(os.path.join(objdir, "nf_bind.o"), tmp_bind)
    # one compiler process per source, at most as many as the CPUs this
    # process may use
    workers = max(1, min(len(cmds), len(os.sched_getaffinity(0)), 8))
    with concurrent.futures.ThreadPoolExecutor(workers) as pool:
        bound = pool.submit(_run, bind[0], verbose) if not isinstance(bind, str) else None
        for f in [pool.submit(_run, c, verbose) for c in cmds]:
            f.result()
    rocm_lib = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(hipcc()))), "lib")
    tmp = LIB + ".tmp"
    _run([hipcc(), "-shared", "-fPIC", *objs, "-o", tmp, f"-Wl,-rpath,{rocm_lib}"], verbose)
    os.replace(tmp, LIB)
    # one of an earlier build would not be this library's
    if os.path.exists(BIND):
        os.remove(BIND)
    if bound is None:
        print(f"no operators on tensors: {bind}", file=sys.stderr)
        return LIB
    bound.result()
    _run(bind[1], verbose)
    os.replace(tmp_bind, BIND)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
