"""Builds libtpq.so (HIP, gfx950) with hipcc and the Python binding's native half with g++, in-tree.

    python -m paper_2411_07942_amd.build            # compile every source, link
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libtpq.so")

SOURCES = ["tpq_api.cpp", "tpq_plan.hip", "tpq_calibrate.hip", "tpq_encode.hip", "tpq_decode.hip", "tpq_gemm.hip",
           "tpq_kv_api.cpp", "tpq_kv.hip", "tpq_kv_attention.hip"]

# -ffp-contract=off: codes, scales and sums must match a non-fused IEEE evaluation.
# -fno-honor-nans: inputs are finite by contract; without it every min / max drags a
# quieting instruction along.  Rounding and evaluation order are unaffected.
# Packed fp32 instructions are switched off (some forms are unreliable on this part).
HIPFLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
            "-fno-honor-nans",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-command-line-argument", "-Wno-unknown-warning-option",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(src: str, extra) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = ["hipcc", "-x", "hip", *HIPFLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines()
                    if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(extra_flags=(), jobs: int = 8) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(lambda s: _compile(s, list(extra_flags)), SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs], check=True)
    os.replace(tmp, LIB)
    build_binding()
    return LIB


BINDING = os.path.join(PKG, "_binding.so")


def build_binding() -> str:
    """The native half of the Python binding: plain C++ against torch's headers, linked to libtpq.so."""
    import sysconfig

    import torch
    t = os.path.dirname(os.path.abspath(torch.__file__))
    tmp = BINDING + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(t, "include"),
           "-isystem", os.path.join(t, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"],
           os.path.join(CSRC, "tpq_binding.cpp"), "-o", tmp,
           "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-L", PKG, "-ltpq",
           "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for tpq_binding.cpp:\n" + r.stderr)
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    os.replace(tmp, BINDING)
    return BINDING


PROBE_SRC = os.path.join(ROOT, "tests", "probes", "hw_probe.hip")
PROBE_BIN = os.path.join(ROOT, "tests", "probes", "hw_probe")


def build_probe() -> str:
    """The stand-alone program that checks the instruction behaviour the kernels rely on
    (run by the GPU tests)."""
    cmd = ["hipcc", "--offload-arch=gfx950", "-O2", "-ffp-contract=off",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-command-line-argument", PROBE_SRC, "-o", PROBE_BIN + ".tmp%d" % os.getpid()]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for hw_probe.hip:\n" + r.stderr)
    os.replace(PROBE_BIN + ".tmp%d" % os.getpid(), PROBE_BIN)
    return PROBE_BIN


if __name__ == "__main__":
    print(build(sys.argv[1:]))
    print(build_probe())
