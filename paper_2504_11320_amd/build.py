"""Build the HIP library (gfx950) in-tree: paper_2504_11320_amd/libwait_sim.so.

Each source is compiled to an object in parallel, then the objects are
linked into one shared library.  Beside it comes _kv.so, the Python module
with the argument checks of the KV-path operators (host code over PyTorch).
The library needs hipcc alone: where what the module needs is not there, or the
module does not compile, it is built all the same."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile
import time
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
SRC_NAMES = ("wait_sim_host.hip", "sim_wait.hip", "sim_fcfs.hip",
             "sim_nested.hip", "sim_nested_unit.hip", "sim_wait_tv.hip", "sim_fcfs_tv.hip",
             "sim_nested_tv.hip", "sim_fcfs_dist.hip", "kv_rows.hip", "kv_attention.hip",
             "kv_norm.hip", "kv_weigh.hip", "kv_evict.hip")
SRCS = [os.path.join(CSRC, f) for f in SRC_NAMES]
INC = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libwait_sim.so")
BINDING = os.path.join(PKG, "_kv.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # identical IEEE operations on both sides of the parity tests
    "-ffp-contract=off", "-fno-fast-math",
    # no packed-FP32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
]


# Instruction-scheduling strategy per translation unit (LLVM's AMDGPU
# scheduler), as measured: the ILP-maximising one against the default is worth
# 1 % on the Nested WAIT kernel for unit thresholds (41.9 against 42.4 ms on the
# heavy-tailed mix), nothing on WAIT (14.52 against 14.47 ms) and costs FCFS 4 %
# (11.87 against 11.44 ms on the chunked mix).
SCHED_FLAGS = {
    "sim_wait.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"],
    "sim_wait_tv.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"],
    "sim_nested_unit.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"],
    "sim_nested.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"],
    "sim_nested_tv.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"],
}


def flags_for(src: str) -> list:
    """hipcc options for one source file."""
    return HIPCC_FLAGS + SCHED_FLAGS.get(os.path.basename(src), [])


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.exists(c) or c == "hipcc"):
            return c
    return "hipcc"


# Host-side AddressSanitizer and UndefinedBehaviorSanitizer (device code is
# built as usual): each -fsanitize= goes right after -Xarch_host.
SANITIZE_FLAGS = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                  "-Xarch_host", "-fno-omit-frame-pointer", "-Xarch_host", "-g"]


def cxx() -> str:
    return os.environ.get("CXX", "g++")


def binding_lacks() -> str:
    """What building the module takes and this machine does not have."""
    lacks = []
    try:
        import torch  # noqa: F401
    except ImportError:
        lacks.append("PyTorch")
    if not os.path.exists(os.path.join(sysconfig.get_path("include"), "Python.h")):
        lacks.append("Python's headers")
    if not shutil.which(cxx()):
        lacks.append(f"a C++ compiler ({cxx()})")
    return ", ".join(lacks)


def build_binding(verbose: bool = False, out: str = BINDING) -> str:
    """Compile the module of csrc/kv_binding.cpp against the installed PyTorch."""
    import torch
    at = os.path.dirname(torch.__file__)
    cmd = [cxx(), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I", INC,
           "-I", sysconfig.get_path("include"), "-isystem", os.path.join(at, "include"),
           "-o", out + ".tmp", os.path.join(CSRC, "kv_binding.cpp"),
           "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(out + ".tmp", out)
    return out


def build(verbose: bool = False, defines=(), out: str = LIB, sanitize: bool = False) -> str:
    """Compile every source for gfx950 and link `out` (default: the in-tree
    library; then the module beside it is compiled too, and an error of that is
    raised once the library is linked).  `defines` are extra -D options;
    `sanitize` instruments the host code with ASan and UBSan (load the result
    with the clang ASan runtime preloaded)."""
    dflags = [f"-D{d}" for d in defines] + (SANITIZE_FLAGS if sanitize else [])
    with tempfile.TemporaryDirectory(prefix="wait_sim_build_") as tmp:
        def compile_one(src: str):
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            cmd = [hipcc()] + flags_for(src) + dflags + ["-I", INC, "-I", CSRC, "-c", "-o", obj, src]
            if verbose:
                print(" ".join(cmd), flush=True)
            t0 = time.perf_counter()
            subprocess.run(cmd, check=True)
            if verbose:
                print(f"  {os.path.basename(src)}: {time.perf_counter() - t0:.1f} s", flush=True)
            return obj

        workers = max(1, min(len(SRCS), os.cpu_count() or 1))
        lacks = binding_lacks() if out == LIB else ""
        with ThreadPoolExecutor(workers) as ex:
            beside = ex.submit(build_binding, verbose, BINDING) if out == LIB and not lacks else None
            objs = list(ex.map(compile_one, SRCS))
        cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", out + ".tmp"] + objs
        if sanitize:
            cmd += ["-fsanitize=address,undefined", "-shared-libasan"]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
    os.replace(out + ".tmp", out)
    failed = beside.exception() if beside else None
    # an earlier build's module may not fit this library
    if (lacks or failed) and os.path.exists(BINDING):
        os.remove(BINDING)
    if failed:
        raise failed
    if lacks:
        print(f"{os.path.basename(BINDING)}, the module behind kv.py, is not built: it takes {lacks}",
              file=sys.stderr, flush=True)
    return out


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
