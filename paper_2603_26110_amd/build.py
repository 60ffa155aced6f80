"""Build libturboesm.so, libturboesm_paged.so and libturboesm_serve.so (HIP, gfx950) in the package directory.

    python -m paper_2603_26110_amd.build

Each source is compiled by hipcc for gfx950 only, without fast-math and with
fp contraction off (the quantizer's binary32 order is part of its contract;
fused multiply-adds are written out explicitly where wanted). Packed fp32
instructions are disabled for the device code.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
OBJ_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libturboesm.so")
LIB_PAGED = os.path.join(PKG, "libturboesm_paged.so")
LIB_SERVE = os.path.join(PKG, "libturboesm_serve.so")
SOURCES = ["tq_api.hip", "tq_quantize.hip", "tq_decode.hip", "tq_dequant.hip", "tq_calibrate.hip",
           "tq_probe.hip"]
# The paged 8-bit cache is a library of its own, with a header of its own.
SOURCES_PAGED = ["paged_api.hip", "paged_pages.hip", "paged_append.hip", "paged_attend.hip"]
# So are the 4-bit one and the operators around it.
SOURCES_SERVE = ["serve_api.hip", "serve_norm.hip", "serve_store.hip", "serve_attend.hip", "serve_verify.hip"]
ARCH = os.environ.get("TQ_OFFLOAD_ARCH", "gfx950")

CFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fno-fast-math", "-fvisibility=hidden",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    path = os.path.join(rocm, "bin", "hipcc")
    return path if os.path.exists(path) else "hipcc"


def _compile(src: str) -> str:
    obj = os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc(), *CFLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    msg = "\n".join(ln for ln in (r.stdout + r.stderr).splitlines() if noise not in ln)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{msg}")
    if msg.strip():
        print(msg, file=sys.stderr)
    return obj


def _link(objs: list[str], lib: str) -> None:
    tmp = lib + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, lib)


def build() -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(_compile, SOURCES + SOURCES_PAGED + SOURCES_SERVE))
    for sources, lib in ((SOURCES, LIB), (SOURCES_PAGED, LIB_PAGED), (SOURCES_SERVE, LIB_SERVE)):
        _link(objs[:len(sources)], lib)
        del objs[:len(sources)]
    return LIB


if __name__ == "__main__":
    print(build())
