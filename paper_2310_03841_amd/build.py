"""Builds libabft.so (HIP kernels + C-ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libabft.so")
SOURCES = ["gemm_tile.hip", "gemm_fast.hip", "gemm_item_rows.hip", "gemm_item_cols.hip", "gemm_item.hip", "gemm_group.hip", "gemm_group_i8.hip", "gemm_group_bf16.hip", "gemm_group_f16.hip", "gemm_group_few.hip", "gemm_group_big_i8.hip", "gemm_group_big_bf16.hip", "gemm_group_big_f16.hip", "gemm_group_big_wgrad.hip", "group_check.hip", "quantize.hip", "aux_kernels.hip", "abft_api.hip"]
HEADERS = ["abft_internal.h", "abft_device.h", "gemm_args.h", "gemm_epilogue.h", "gemm_apass.h", "gemm_item.h", "block_out.h", "encode_pass.h", "predict_pass.h", "check_dots.h", "gemm_fast_tile.h", "group_args.h", "gemm_group.h", "gemm_group_big.h", "group_passes.h", os.path.join("..", "..", "include", "abft.h")]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17", "-munsafe-fp-atomics",
    # packed fp32 instructions are kept out of generated code on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


# The fast GEMM kernels count their outstanding loads by hand and keep up to 128 accumulators per lane, two waves to a SIMD:
# a register spilled to scratch memory inside them costs speed at best.  The build fails on one.
NO_SPILL_SOURCES = ["gemm_fast.hip", "gemm_group_big_i8.hip", "gemm_group_big_bf16.hip", "gemm_group_big_f16.hip", "gemm_group_big_wgrad.hip"]


def _check_no_spills(remarks: str) -> None:
    name = None
    for line in remarks.splitlines():
        if "Function Name:" in line:
            name = line.split("Function Name:")[1].split()[0]
        elif "ScratchSize [bytes/lane]:" in line and name and ("gemm_fast_kernel" in name or "gemm_group_big_kernel" in name):
            size = int(line.split("ScratchSize [bytes/lane]:")[1].split()[0])
            if size != 0:
                raise RuntimeError(f"{name} spills {size} bytes per lane to scratch memory")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    hdrs = [os.path.normpath(os.path.join(CSRC, h)) for h in HEADERS]
    jobs = []
    objs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".hip", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + hdrs):
            extra = ["-Rpass-analysis=kernel-resource-usage"] if src in NO_SPILL_SOURCES else []
            jobs.append(["hipcc", *FLAGS, *extra, "-c", s, "-o", o])

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("hipcc failed: " + " ".join(cmd))
        return r.stderr

    with ThreadPoolExecutor(max_workers=8) as ex:
        logs = list(ex.map(run, jobs))
    for cmd, log in zip(jobs, logs):
        if "-Rpass-analysis=kernel-resource-usage" in cmd:
            _check_no_spills(log)
    if jobs or not os.path.exists(LIB):
        run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs])
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
