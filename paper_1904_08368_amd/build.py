"""Compile the HIP sources into librelayfused.so (gfx950 only), in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librelayfused.so")
SOURCES = ["api.cpp", "api_attention.cpp", "fusion.cpp", "launch_list.cpp", "conv_block.hip", "conv_group.hip", "conv_igemm.hip", "conv_igemm_dma.hip", "conv_halo.hip", "conv_small.hip", "conv_stream.hip", "conv_direct_f32.hip", "conv_first.hip", "conv_stem.hip", "head.hip", "dwconv.hip", "dwpw.hip", "dwpw_direct.hip", "dense.hip", "glue.hip", "quant.hip", "realize.hip", "probe.hip", "qschemes.hip", "rope.hip", "paged_attention.hip", "paged_attention_tiles.hip", "dense_w4.hip", "api_decoder.cpp", "norm.hip", "route.hip", "sample.hip", "experts_w4.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # a kernel's leading scalar parameters are in registers when a wave starts (see xcd_remap)
         "-mllvm", "-amdgpu-kernarg-preload-count=16",
         "-Wall", "-Wno-unused-command-line-argument"]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for src in SOURCES:
        obj = os.path.join(HERE, "_build", src + ".o")
        cmd = [hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        # the host pass warns that it does not know the packed-fp32 feature: harmless
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l and l.strip())
        if p.returncode != 0:
            failed = True
            print(f"[build] {src} FAILED\n{out}", file=sys.stderr)
        elif out and verbose:
            print(f"[build] {src}:\n{out}")
    if failed:
        raise RuntimeError("hipcc failed")
    # link beside the target and rename: a process that has the old library mapped keeps a valid file
    tmp = LIB + ".tmp"
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs], check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
