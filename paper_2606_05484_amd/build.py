"""Compile libmapl.so for gfx950 in-tree (hipcc, no JIT, no torch extension).

    python -m paper_2606_05484_amd.build          # or build() from Python

Objects go to _build/ at the repository root; the shared library lands next
to this file as libmapl.so.  Every HIP source is compiled with the packed
fp32 feature disabled (the host pass warns that it does not know the
feature; that warning is harmless).
"""
import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libmapl.so")
ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCES = ["k_gemm_bf16.hip", "k_gemm_deep.hip", "k_gemm_f32.hip", "k_gemm_f32s.hip", "k_sym.hip", "k_wgrad.hip", "k_rvq.hip", "k_prep.hip", "k_misc.hip",
           "k_anchor.hip", "k_grvq.hip", "k_ckpt.hip", "k_xent.hip", "k_norm_fwd.hip", "k_norm_bwd.hip", "k_norm_bwd_f32.hip", "k_optim.hip",
           "mapl_api.cpp"]
FLAGS = ["--offload-arch=%s" % ARCH, "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include")]


# Per-file flags: the RVQ kernels keep their accumulators in ordinary VGPRs
# (their score folds read every accumulator element; the AGPR form would add
# a copy per element).
EXTRA = {f: ["-mllvm", "-amdgpu-mfma-vgpr-form=1"] for f in ("k_rvq.hip", "k_grvq.hip")}


def _compile(src):
    obj = os.path.join(BUILD, src + ".o")
    cmd = [HIPCC] + FLAGS + EXTRA.get(src, []) + ["-c", os.path.join(CSRC, src), "-o", obj]
    if src.endswith(".cpp"):
        cmd[1:1] = ["-x", "hip"]
    p = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    msg = "\n".join(l for l in (p.stdout + p.stderr).splitlines() if noise not in l)
    if p.returncode != 0:
        raise RuntimeError("hipcc failed on %s:\n%s" % (src, msg))
    return obj, msg


def build(verbose=False):
    os.makedirs(BUILD, exist_ok=True)
    jobs = min(len(SOURCES), max(1, int(os.environ.get("MAX_JOBS", os.cpu_count() or 4))))
    with cf.ThreadPoolExecutor(jobs) as ex:
        results = list(ex.map(_compile, SOURCES))
    for _, msg in results:
        if verbose and msg.strip():
            print(msg)
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=%s" % ARCH, "-shared", "-fPIC", "-o", tmp] + [o for o, _ in results]
    p = subprocess.run(cmd, capture_output=True, text=True)
    if p.returncode != 0:
        raise RuntimeError("link failed:\n" + p.stdout + p.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
