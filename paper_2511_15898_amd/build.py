"""Build step: compiles the HIP sources of the verifier into one shared library for gfx950."""
from __future__ import annotations

import os
import subprocess

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
LIB_PATH = os.path.join(PKG_DIR, "libgr_verify.so")
SOURCES = ["gr_select.hip", "gr_solve.hip", "gr_full.hip", "gr_sweep.hip", "gr_grid.hip", "gr_verify.hip", "gr_rows.hip", "gr_draft.hip", "gr_beam.hip",
           "gr_pages.hip", "gr_api.hip"]


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG_DIR, "csrc")]
    cmd += [os.path.join(PKG_DIR, "csrc", s) for s in SOURCES]
    cmd += ["-o", LIB_PATH]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
