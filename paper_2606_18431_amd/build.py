"""Build the HIP libraries for gfx950 with hipcc, in-tree: libtas.so;
libtas_check.so, the same entry points with every batch, every run of
repeated iterations and every instance's state verified (TAS_CHECK_INVARIANTS);
and libtas_step.so, the operators of a serving iteration (tas_step.h, tas_fp4.h)."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libtas.so")
CHECK_LIB = os.path.join(PKG, "libtas_check.so")
STEP_LIB = os.path.join(PKG, "libtas_step.so")
SOURCES = ["tas_abi.hip", "tas_sim.hip", "tas_pctl.hip", "tas_order.hip"]
STEP_SOURCES = ["tas_step_abi.hip", "tas_step_append.hip", "tas_step_attn.hip",
                "tas_fp4_abi.hip", "tas_fp4_append.hip", "tas_fp4_attn.hip", "tas_fp4_pack.hip",
                "tas_fp4_linear.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _command(out: str, sources: list[str], flags: list[str]) -> list[str]:
    srcs = [os.path.join(CSRC, s) for s in sources]
    return [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC] + flags + ["-o", out] + srcs


def build(verbose: bool = False) -> str:
    """Compile every HIP source into libtas.so, libtas_check.so and
    libtas_step.so (always recompiles; the builds run side by side). Returns
    libtas.so's path."""
    # every floating-point step of the adaptive gamma is one rounded IEEE
    # operation, as in its definition: no fused multiply-add
    exact = ["-ffp-contract=off"]
    jobs = [(LIB, SOURCES, exact), (CHECK_LIB, SOURCES, exact + ["-DTAS_CHECK_INVARIANTS=1"]),
            (STEP_LIB, STEP_SOURCES, [])]
    procs = []
    for out, sources, flags in jobs:
        cmd = _command(out + ".tmp", sources, flags)
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((out, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
    failed = False
    for out, p in procs:
        log, _ = p.communicate()
        if p.returncode != 0:
            sys.stderr.write(log)
            failed = True
        else:
            os.replace(out + ".tmp", out)
    if failed:
        raise RuntimeError("hipcc failed")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
