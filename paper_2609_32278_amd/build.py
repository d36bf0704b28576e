"""Build libkvx.so (HIP kernels + host C ABI) for gfx950 with hipcc, in-tree."""

from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libkvx.so")

ARCH = "gfx950"
# Packed fp32 VALU ops are disabled for all device code (-packed-fp32-ops).
# MFMA results go to ordinary VGPRs (the attention kernel keeps its score tiles,
# which the softmax works on, out of AGPRs that would need copies back).
HIP_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Wall",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-mllvm", "-amdgpu-mfma-vgpr-form=true",
             "-I", INCLUDE, "-I", CSRC]

# The scheduler's own count of live registers, for the prefill kernels of 8-bit pools in their
# exact form: at 244 to 256 VGPRs the generic one overcounts three of their four unrolled
# iterations and lines the products up without anything beside them (1064 against 1156 TFLOP/s).
EXTRA_FLAGS = {name: ["-mllvm", "-amdgpu-use-amdgpu-trackers=1"]
               for name in ("kvx_page_attn.hip", "kvx_cross.hip", "kvx_cross_page.hip")}


def hipcc() -> str:
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found; ROCm is required to build libkvx")
    return path


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def build(verbose: bool = False) -> str:
    """Compile every source (in parallel) and link libkvx.so next to this file."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    cc = hipcc()
    procs = []
    objs = []
    for src in sources():
        obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
        objs.append(obj)
        cmd = [cc, *HIP_FLAGS, *EXTRA_FLAGS.get(os.path.basename(src), []), "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        noise = [ln for ln in out.splitlines() if "packed-fp32-ops" not in ln]
        if p.returncode != 0:
            failed.append((src, "\n".join(noise)))
        elif verbose and noise:
            print("\n".join(noise), flush=True)
    if failed:
        msg = "\n\n".join(f"{s}:\n{o}" for s, o in failed)
        raise RuntimeError(f"hipcc failed:\n{msg}")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [cc, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *objs]
    subprocess.run(cmd, check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
