"""Builds libdistgrid.so (HIP, gfx950 only) in-tree with hipcc.  Run: python -m paper_2405_04416_amd.build"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libdistgrid.so")
PEAKS_PATH = os.path.join(HERE, "libdgpeaks.so")     # yardstick kernels of the benchmark, not part of the library

SOURCES = ["host.hip", "segments.hip", "encode.hip", "encode_bwd_binned.hip", "encode_bwd_fill.hip", "order.hip", "encode_ordered.hip", "mlp.hip", "mlp_mfma.hip", "mlp_small.hip", "render.hip", "optim.hip", "occupancy.hip",
           "norm.hip", "recurrence.hip", "dropout.hip", "rms_norm.hip", "rows_e4m3.hip", "product_e4m3.hip",
           "delta.hip", "delta_token.hip", "delta_small.hip", "delta_weights.hip", "delta_fwd.hip", "delta_bwd.hip", "delta_join.hip", "delta_grad.hip"]
COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
          # packed fp32 instructions are kept out of every kernel of this library
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC]
PER_FILE = {"segments.hip": ["-ffp-contract=off"], "occupancy.hip": ["-ffp-contract=off"]}   # bit-exact fp32 bookkeeping: no fused multiply-add
# sums of matrix instructions in the registers that the other instructions use: without copies between them these two take a tenth less time
PER_FILE.update({name: ["-mllvm", "-amdgpu-mfma-vgpr-form=1"] for name in ("delta_fwd.hip", "delta_bwd.hip")})


def hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("hipcc not found")


def _compile(src):
    obj = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
    cmd = [hipcc(), "-c", os.path.join(CSRC, src), "-o", obj] + COMMON + PER_FILE.get(src, [])
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops"     # the host pass does not know this device feature; harmless
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, res.stderr))
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_library(verbose=True):
    """Compiles every source and links the shared library; always rebuilds."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as pool:
        objs = list(pool.map(_compile, SOURCES + ["peaks.hip"]))
    for path, members in ((LIB_PATH, objs[:-1]), (PEAKS_PATH, objs[-1:])):
        cmd = [hipcc(), "-shared", "-fPIC", "--offload-arch=gfx950", "-o", path] + members
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("link failed:\n" + res.stderr)
        if verbose:
            print("built", path)
    return LIB_PATH


if __name__ == "__main__":
    build_library()
