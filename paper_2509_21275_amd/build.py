"""Compiles the HIP sources under csrc/ into libchunk_attn.so (gfx950) with hipcc."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libchunk_attn.so")
SOURCES = ["plan.cpp", "chunk_plan.cpp", "chunk_sched.cpp", "fused_ce.hip", "chunk_rope.hip", "fused_norm.hip", "chunk_linear.hip", "paged_cache.hip", "paged_attn.hip", "draft_verify.hip", "fwd_kernel.hip", "bwd_kernel.hip", "bwd_fused_kernel.hip", "bwd_share_kernel.hip", "measure.hip", "api.hip"]
# -packed-fp32-ops off: the compiler must not form packed fp32 VALU instructions on this target
# -fno-honor-nans: no input of these kernels is NaN; it lets max/compare lower to single instructions
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function", "-fno-honor-nans",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# ... but for those that say what becomes of a NaN
HONOR_NANS = {"paged_cache.hip", "paged_attn.hip", "draft_verify.hip"}


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(bdir, os.path.splitext(src)[0] + ".o")
        cmd = [hipcc, *FLAGS, *(["-fhonor-nans"] if src in HONOR_NANS else []), "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{msgs}")
        if verbose and msgs.strip():
            print(msgs)
        return obj

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + f".tmp{os.getpid()}"
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
