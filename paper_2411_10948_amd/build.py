"""Build libshiftquant.so (HIP, gfx950) in-tree with hipcc.

Usage: python -m paper_2411_10948_amd.build [-v]
"""
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libshiftquant.so")
SOURCES = ["sq_abi.hip", "sq_quant.hip", "sq_gemm.hip", "sq_l1bn.hip", "sq_mx_abi.hip", "sq_mx.hip",
           "sq_mx_gemm.hip", "sq_act.hip", "sq_block_abi.hip", "sq_norm.hip", "sq_route.hip", "sq_exchange.hip",
           "sq_f8_abi.hip", "sq_f8.hip", "sq_f8_gemm.hip"]
ARCH = "gfx950"

HIPCC_FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    # IEEE fp32: no FMA contraction, correctly rounded division, denormals kept
    "-ffp-contract=off",
    "-fhip-fp32-correctly-rounded-divide-sqrt",
    "-fno-gpu-flush-denormals-to-zero",
    # never emit packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA accumulators in VGPRs: with the accumulator-register form the
    # compiler copied every accumulator into and out of AGPRs around each
    # MFMA (four copies per 16x16x64 instruction in the streaming kernels)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-mcode-object-version=5",
    "-Wall",
    # every symbol resolved at link time (a kernel whose host stub went
    # missing must fail the build, not the first launch)
    "-Wl,--no-undefined",
]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False) -> str:
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    tmp = LIB + ".tmp"
    cmd = [hipcc(), *HIPCC_FLAGS, f"-I{INCLUDE}", f"-I{CSRC}", *srcs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass warns that it does not know the packed-fp32 feature
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
