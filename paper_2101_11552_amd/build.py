"""Builds libtfg.so (the HIP library behind include/tfg.h) and libtfg_probe.so
(the benchmark's gather probes, include/tfg_probe.h) for gfx950 in-tree.

Every translation unit is compiled by hipcc to an object file (in parallel),
then linked into a shared library next to this file.
"""

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libtfg.so")
# (the longest to compile first)
SOURCES = ["attention_grad_f32_wide.hip", "attention_grad_bf16_wide.hip",
           "attention_grad_f32_narrow.hip", "attention_grad_bf16_narrow.hip",
           "attention_f32_wide.hip", "attention_bf16_wide.hip",
           "attention_f32_narrow.hip", "attention_bf16_narrow.hip",
           "csr.hip", "norm.hip", "aggregate.hip", "slots_sum.hip", "slots_max.hip",
           "slots_heads.hip", "slots_masked.hip", "softmax.hip",
           "gat.hip", "gat_dot.hip", "pool.hip", "batch.hip", "backward.hip",
           "embed.hip", "group_norm.hip", "attention.hip", "attention_grad.hip", "api.cpp"]
# measurement probes for the benchmark (include/tfg_probe.h), a library of their own
PROBE_LIB = os.path.join(HERE, "libtfg_probe.so")
PROBE_SOURCES = ["probe.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # keep the compiler from emitting packed-fp32 arithmetic
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix products keep their sums in ordinary registers, where the softmax reads them
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-I", os.path.join(ROOT, "include"),
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [HIPCC, *FLAGS, *lang, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def _link(objs, lib: str) -> None:
    tmp = lib + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = SOURCES + PROBE_SOURCES
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    _link(objs[:len(SOURCES)], LIB)
    _link(objs[len(SOURCES):], PROBE_LIB)
    if verbose:
        print(LIB)
        print(PROBE_LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
