"""Builds libstq.so (the C-ABI library) in-tree with nvcc for sm_100a, and _lists.so (a Python module over torch's headers)."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libstq.so")
LISTS, LISTS_SOURCE = os.path.join(HERE, "_lists.so"), os.path.join(CSRC, "stq_lists.cpp")
SOURCES = ["stq_step_fast.cu", "stq_step_variants.cu", "stq_step_split.cu", "stq_kernels.cu", "stq_static_stats.cu",
           "stq_q8_rows.cu", "stq_q8_linear.cu", "stq_q8_grad.cu", "stq_q8_tma.cpp", "stq_q8_api.cu",
           "stq_vocab_scores.cu", "stq_vocab_grad.cu", "stq_vocab_api.cu", "stq_clip.cu",
           "stq_api.cu", "stq_policy.cpp"]
HEADERS = [os.path.join(CSRC, "stq_internal.h"), os.path.join(CSRC, "stq_handle.h"), os.path.join(CSRC, "stq_q8.h"),
           os.path.join(CSRC, "stq_q8_mma.cuh"), os.path.join(CSRC, "stq_q8_tma.h"), os.path.join(CSRC, "stq_q8_ring.h"),
           os.path.join(CSRC, "stq_checks.h"), os.path.join(CSRC, "stq_rowcopy.cuh"), os.path.join(CSRC, "stq_vocab.h"),
           os.path.join(CSRC, "stq_vocab_ranges.h"), os.path.join(CSRC, "stq_step_fast.cuh"), os.path.join(os.path.dirname(HERE), "include", "stq.h")]

# -fmad=false: the code-deciding arithmetic must not be contracted; fused operations are written
# explicitly where they are wanted.
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo", "--threads", "0",
    "-fmad=false", "-Xcompiler", "-fPIC", "-shared", "-cudart", "static",
    "-diag-suppress", "177",     # unused members of the per-width constant tables
]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def older(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def stale() -> bool:
    return older(LIB, [os.path.join(CSRC, s) for s in SOURCES] + HEADERS)


def build_lists(force: bool = False) -> str:
    if not force and not older(LISTS, [LISTS_SOURCE, HEADERS[-1]]):
        return LISTS
    torch_dir = os.path.dirname(importlib.util.find_spec("torch").origin)
    inc, tmp = os.path.join(torch_dir, "include"), LISTS + f".tmp{os.getpid()}"
    subprocess.check_call([
        "g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-I{inc}", f"-I{inc}/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}",
        "-o", tmp, LISTS_SOURCE, f"-L{torch_dir}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, LISTS)
    return LISTS


def build(force: bool = False, verbose: bool = False) -> str:
    build_lists(force)
    if not force and not stale():
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-o", tmp,
           *[os.path.join(CSRC, s) for s in SOURCES]]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
