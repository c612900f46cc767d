"""Builds libstq.so (the C-ABI library) in-tree with nvcc for sm_100a, and _lists_torch_* (a Python module over torch's headers, for the torch
and the Python that are there)."""
from __future__ import annotations

import os
import re
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libstq.so")
LISTS_SOURCE = os.path.join(CSRC, "stq_lists.cpp")
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


def lists_name(torch_version: str) -> str:
    """The module's name: it reads torch's objects in place, so each version has its own."""
    return "_lists_torch_" + re.sub(r"\W", "_", torch_version)


def build_lists(force: bool = False) -> str | None:
    try:
        import torch
    except ImportError:
        print("torch is not there: the module for lists of tensors is not built (clip.py needs it, libstq does not)", file=sys.stderr)
        return None
    name = lists_name(torch.__version__)
    target = os.path.join(HERE, name + sysconfig.get_config_var("EXT_SUFFIX"))
    if not force and not older(target, [LISTS_SOURCE, HEADERS[-1]]):
        return target
    torch_dir, tmp = os.path.dirname(torch.__file__), target + f".tmp{os.getpid()}"
    inc = os.path.join(torch_dir, "include")
    subprocess.check_call([
        "g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-DSTQ_LISTS={name}", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
        f"-I{inc}", f"-I{inc}/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}",
        "-o", tmp, LISTS_SOURCE, f"-L{torch_dir}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, target)
    return target


def build_lib(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-o", tmp,
           *[os.path.join(CSRC, s) for s in SOURCES]]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


def build(force: bool = False, verbose: bool = False) -> str:
    lib = build_lib(force, verbose)
    build_lists(force)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
