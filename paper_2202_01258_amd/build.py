"""Builds the HIP libraries for gfx950: libqd.so, the MAP-Elites generation, and
libqdseq.so, the operators of sequence policies.

hipcc cross-compiles without a GPU.  Flags that the arithmetic of libqd.so relies on:
  -ffp-contract=off                      no fused multiply-add except explicit ones
  -fhip-fp32-correctly-rounded-divide-sqrt   IEEE division and square root
  -Xclang -target-feature -Xclang -packed-fp32-ops   no packed fp32 instructions (both libraries)
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libqd.so")
SRC = [os.path.join(HERE, "csrc", "qd_lib.hip")]
DEPS = SRC + [os.path.join(HERE, "csrc", f) for f in ("qd_device.hpp", "qd_kernels.hpp",
                                                       "qd_rollout.hpp")] + [
    os.path.join(ROOT, "include", "qd.h")]
SEQ_LIB = os.path.join(HERE, "libqdseq.so")
SEQ_SRC = [os.path.join(HERE, "csrc", f) for f in ("seq_norm.hip", "seq_window.hip",
                                                   "seq_decay.hip", "seq_conv.hip", "seq_scan.hip",
                                                   "seq_scan_backward.hip", "seq_branch.hip", "seq_dropout.hip")]
SEQ_DEPS = SEQ_SRC + [os.path.join(HERE, "csrc", f) for f in ("seq_common.hpp", "seq_plan.hpp", "seq_rows.hpp",
                                                                  "seq_scan.hpp")] + [
    os.path.join(ROOT, "include", "qd_seq.h")]
ARCH = os.environ.get("QD_OFFLOAD_ARCH", "gfx950")


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def flags() -> list[str]:
    return [
        f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
        "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-Wall", "-Wno-unused-result", "-Wno-unused-function",
    ]


def build(verbose: bool = False, extra: list[str] | None = None) -> str:
    tmp = LIB + ".tmp"
    cmd = [hipcc(), *flags(), *(extra or []), *SRC, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


def seq_flags() -> list[str]:
    return [
        f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-Wall", "-Wno-unused-result", "-Wno-unused-function",
    ]


def build_seq(verbose: bool = False, extra: list[str] | None = None) -> str:
    """libqdseq.so: its sources compiled side by side, then linked."""
    with tempfile.TemporaryDirectory() as tmp:
        objects, running = [], []
        for src in SEQ_SRC:
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            cmd = [hipcc(), *seq_flags(), *(extra or []), "-c", src, "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            objects.append(obj)
            running.append((cmd, subprocess.Popen(cmd)))
        failed = [cmd for cmd, p in running if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        out = SEQ_LIB + ".tmp"
        subprocess.run([hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objects, "-o", out],
                       check=True)
    os.replace(out, SEQ_LIB)
    return SEQ_LIB


if __name__ == "__main__":
    build(verbose=True, extra=[a for a in sys.argv[1:] if a != "-v"])
    build_seq(verbose=True, extra=[a for a in sys.argv[1:] if a != "-v"])
