"""Builds libvsprefill.so (hand-written HIP for gfx950) in-tree with hipcc."""
import glob
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libvsprefill.so")
SOURCES = sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))
HEADERS = sorted(glob.glob(os.path.join(HERE, "csrc", "*.h"))) + [os.path.join(ROOT, "include", "vsprefill.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    "-ffp-contract=off",
    # packed fp32 VALU forms are switched off: some of them have given wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"),
]
# per-source additions
EXTRA_FLAGS = {
    # one wavefront per SIMD with 512 registers: score accumulators go to the vector registers the softmax reads
    "vs_dense.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    # the same: 280 fewer register copies per 32-token block
    "vs_train.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    # score and output accumulators in the registers that the conversions and the softmax use
    "vs_cache_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "vs_cache_tile.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "vs_cache_prefill.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "vs_cache_weigh.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
}


def stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in SOURCES + HEADERS)


def build_library(force=True, verbose=False):
    """Compile every .hip source and link the shared library.  Returns its path."""
    if not force and not stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    for src in SOURCES:
        obj = os.path.join(bdir, os.path.basename(src) + ".o")
        objs.append(obj)
        cmd = [hipcc] + HIPCC_FLAGS + EXTRA_FLAGS.get(os.path.basename(src), []) + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd))
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, pr in procs:
        out, _ = pr.communicate()
        if pr.returncode != 0:
            raise RuntimeError("hipcc failed on %s:\n%s" % (src, out))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
