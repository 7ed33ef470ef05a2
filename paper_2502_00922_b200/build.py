"""Build libhuffllm.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(os.path.dirname(PKG), "include")
SO = os.path.join(PKG, "libhuffllm.so")
SOURCES = ["host_codec.cpp", "api.cu", "kernels.cu", "kernels_epilogue.cu", "kernels_tc.cu", "kernels_tc_epilogue.cu", "kernels_tc_epilogue_fp16.cu",
           "norm.cu", "split_explorer.cu", "encode_device.cu"]


def needs_build() -> bool:
    if not os.path.exists(SO):
        return True
    t = os.path.getmtime(SO)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "huffllm.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return SO
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-I" + INCLUDE, "-Xcompiler", "-fPIC"]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    with tempfile.TemporaryDirectory() as tmp:       # one compiler per source, side by side
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        running = [subprocess.Popen(cmd + ["-c", "-o", o, os.path.join(CSRC, s)]) for s, o in zip(SOURCES, objects)]
        failed = [s for s, p in zip(SOURCES, running) if p.wait() != 0]
        if failed:
            raise RuntimeError("nvcc failed on " + ", ".join(failed))
        subprocess.check_call(cmd + ["-shared", "-o", SO] + objects + ["-lpthread"])
    return SO


if __name__ == "__main__":
    print(build(force=True, verbose=True))
