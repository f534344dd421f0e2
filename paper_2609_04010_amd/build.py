"""Build libdd.so (the gfx950 HIP library behind include/dd.h) in-tree with hipcc.

Usage: python -m paper_2609_04010_amd.build [-v]
"""
import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdd.so")

SOURCES = ["dd_api.hip", "k_posterior.hip", "k_latent_init.hip", "k_norm.hip", "k_gemm.hip",
           "k_gemm_ring.hip",
           "k_attn.hip", "k_verify.hip", "k_cache.hip", "k_cache_attn.hip", "k_edit.hip"]

# Per-file extra flags.  Attention keeps its MFMA accumulators in ordinary VGPRs (the softmax reads
# every score with VALU instructions; AGPR accumulators would need a copy per score).  The GEMMs need
# the AGPR file for their 256 accumulators and keep the default.
EXTRA = {f: ["-mllvm", "-amdgpu-mfma-vgpr-form"] for f in ("k_attn.hip", "k_cache_attn.hip")}

FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
         # packed-FP32 instructions stay off everywhere: some of their forms have given wrong results
         # on this hardware without any error
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC,
         "-Wno-unused-result"]


def _hipcc():
    h = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(h):
        raise RuntimeError("hipcc not found")
    return h


def _compile(src, verbose):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc(), *FLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = (r.stdout + r.stderr)
    # the host pass does not know the packed-fp32 feature and says so; that line is noise
    out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{out}")
    if verbose and out.strip():
        print(out)
    return obj


def build(verbose=False):
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), "-shared", "--offload-arch=gfx950", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
