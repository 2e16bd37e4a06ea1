"""Builds liboptimus.so (HIP, gfx950 only) in-tree with hipcc.  No JIT, no torch extension machinery:
the library is a plain C-ABI shared object."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "liboptimus.so")
SOURCES = ["api.hip", "gemm_mfma.hip", "gemm_mfma_ragged.hip", "gemm_mfma_deep.hip", "gemm_mfma_pair64.hip", "gemm_mfma_pair128.hip", "gemm_generic.hip", "gemm_short.hip", "layernorm.hip", "softmax.hip", "attention_fused.hip", "attention_fused_wide.hip", "attention_probs.hip", "attention_biased.hip", "attention_biased_bwd.hip", "blocks.hip", "stack.hip", "model_ends.hip", "adamw.hip", "attention_select.hip", "attention_selected.hip", "attention_selected_bwd.hip", "attention_selected_masked.hip", "rotary.hip", "gradients.hip", "probe.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(CSRC, src.replace(".hip", ".o"))
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build_library(verbose: bool = False) -> str:
    """Compile every source and link the shared library; always rebuilds."""
    with ThreadPoolExecutor(max_workers=min(6, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build_library(verbose=True)
