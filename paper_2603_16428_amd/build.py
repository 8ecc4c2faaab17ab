"""Builds the HIP library of the fused linear + cross-entropy step for gfx950.

    python -m paper_2603_16428_amd.build

compiles csrc/lce_api.hip (which includes the step's kernels), csrc/ops_api.hip (the operators around
the step), csrc/embedding_api.hip, csrc/mxfp4_api.hip and csrc/sample_api.hip (those on the vocabulary's matrix and
logits) and csrc/host_adam.cpp (the host optimizer step) into liblce.so next to this file.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "liblce.so")
KERNEL_SOURCES = [os.path.join(HERE, "csrc", "lce_api.hip")]
OPS_SOURCES = [os.path.join(HERE, "csrc", "ops_api.hip")]
VOCAB_SOURCES = [os.path.join(HERE, "csrc", name) for name in ("embedding_api.hip", "mxfp4_api.hip", "sample_api.hip")]
HOST_SOURCES = [os.path.join(HERE, "csrc", "host_adam.cpp")]
SOURCES = KERNEL_SOURCES + OPS_SOURCES + VOCAB_SOURCES + HOST_SOURCES
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # No packed fp32 arithmetic in device code.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


# Host-only C++ (the optimizer step: function multiversioning and x86 _Float16, which the HIP
# compile of a .cpp would also try to build for the GPU) goes through the host compiler first.
HOSTCXX = os.environ.get("LCE_HOSTCXX", "/opt/rocm/llvm/bin/clang++")
HOST_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-I", os.path.join(ROOT, "include")]


def build(verbose: bool = False) -> str:
    """Compile liblce.so (always) and return its path. Raises on failure."""
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as d:
        # One compiler process per source, at the same time.
        device = [HIPCC] + [f for f in FLAGS if f != "-shared"]
        objs, started = [], []
        for src in SOURCES:
            obj = os.path.join(d, os.path.splitext(os.path.basename(src))[0] + ".o")
            objs.append(obj)
            cmd = ([HOSTCXX] + HOST_FLAGS if src in HOST_SOURCES else device) + ["-c", src, "-o", obj]
            started.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        ended = [(cmd, p.communicate()[0], p.returncode) for cmd, p in started]
        if all(rc == 0 for _, _, rc in ended):
            cmd = [HIPCC] + FLAGS + objs + ["-pthread", "-o", tmp]
            r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            ended.append((cmd, r.stdout, r.returncode))
    msgs = [ln for _, out, _ in ended for ln in out.splitlines() if "packed-fp32-ops" not in ln]
    failed = [" ".join(cmd) for cmd, _, rc in ended if rc != 0]
    if failed:
        raise RuntimeError("failed: " + "; ".join(failed) + "\n" + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs), file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
