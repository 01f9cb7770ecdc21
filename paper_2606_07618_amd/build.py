"""Build step: compile the HIP library for gfx950 in-tree (libnvfp4ss.so beside this file)."""
from __future__ import annotations

import os
import subprocess
from pathlib import Path

HERE = Path(__file__).resolve().parent
ROOT = HERE.parent
SRC = HERE / "csrc" / "nvfp4ss.hip"
SOURCES = [SRC, HERE / "csrc" / "optimum.hip", HERE / "csrc" / "importance.hip",
           HERE / "csrc" / "gptq.hip", HERE / "csrc" / "mxfp4.hip", HERE / "csrc" / "matmul.hip",
           HERE / "csrc" / "ffn.hip"]
LIB = HERE / "libnvfp4ss.so"

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                                # no fusion beyond the written fmaf
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def build(out: Path = LIB, verbose: bool = False) -> Path:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, *HIPCC_FLAGS, f"-I{ROOT / 'include'}", "-o", str(out), *map(str, SOURCES)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed:\n{r.stdout}\n{r.stderr}")
    if verbose and r.stderr.strip():
        print(r.stderr)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
