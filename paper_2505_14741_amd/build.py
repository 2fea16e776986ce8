"""Build the HIP C-ABI library for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libparastep_hip.so")
SOURCES = ["api.hip", "elementwise.hip", "gemm.hip", "gemm_mfma.hip", "gemm_few.hip", "slim.hip", "attention.hip", "probe.hip",
           "cross_attention.hip", "gemm_fp8.hip", "group_norm.hip", "gemm_fp4.hip", "qk_norm.hip", "packed_attention.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument",
         # an access wider than its address allows is an error: the hardware may take it, the compiler need not
         "-Werror=align-mismatch"]


# per-file additions: the attention loop is a long straight-line mix of matrix, vector and LDS instructions at the
# register limit; of the compiler's scheduling strategies (same instructions, same results) iterative-minreg orders it
# fastest: against the default 1.2 % at 17776 keys, against max-ilp 0.5 % (1 % at 33976 keys, 2 % for the kernel that
# tracks a softmax reference); iterative-ilp is 8 % slower
FILE_FLAGS = {"attention.hip": ["-mllvm", "-amdgpu-sched-strategy=iterative-minreg"]}


def _compile(src: str, extra) -> str:
    obj = os.path.join(CSRC, "_build", src.replace(".hip", ".o"))
    os.makedirs(os.path.dirname(obj), exist_ok=True)
    cmd = [HIPCC, *FLAGS, *FILE_FLAGS.get(src, []), *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    warn = [l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l and l.strip()]
    if warn and os.environ.get("PS_BUILD_VERBOSE"):
        print("\n".join(warn), file=sys.stderr)
    return obj


def build_library(extra_flags=()) -> str:
    with ThreadPoolExecutor(max_workers=min(len(SOURCES), 6)) as ex:
        objs = list(ex.map(lambda s: _compile(s, list(extra_flags)), SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    return LIB


if __name__ == "__main__":
    print(build_library(sys.argv[1:]))
