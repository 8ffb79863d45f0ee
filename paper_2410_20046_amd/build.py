"""Builds libdqrm.so (the gfx950 HIP kernels + C ABI) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libdqrm.so")
_SHARED = ["dqrm_host.hpp", "dqrm_fastdiv.hpp", os.path.join(ROOT, "include", "dqrm.h")]
# each translation unit and the headers it includes
UNITS = {
    "dqrm_api.hip": ["dqrm_device.hpp", "dqrm_fwd.hpp", "dqrm_dedupe.hpp", "dqrm_bwd.hpp", "dqrm_update.hpp", "dqrm_merge.hpp",
                     "dqrm_dense.hpp", "dqrm_step.hpp"] + _SHARED,
    "dqrm_mx_api.hip": ["dqrm_mx.hpp", "dqrm_mx_gemm.hpp", "dqrm_mx_few.hpp", "dqrm_norm.hpp"] + _SHARED,
}
SOURCES = [os.path.join(CSRC, f) for f in UNITS]
HEADERS = sorted({os.path.join(CSRC, f) for headers in UNITS.values() for f in headers})

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # results are compared bit for bit with a CPU oracle: one rounding per
    # operation, correctly rounded fp32 division
    "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt",
    # do not let the compiler form packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    m = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > m for f in SOURCES + HEADERS)


def build_library(force: bool = True, verbose: bool = False) -> str:
    """Compile the library, its translation units side by side.  Cross-compiles for gfx950; needs no GPU."""
    if not force and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objects, running = [], []
    for unit, headers in UNITS.items():
        source = os.path.join(CSRC, unit)
        obj = os.path.splitext(source)[0] + ".o"
        objects.append(obj)
        newest = max(os.path.getmtime(os.path.join(CSRC, f)) for f in [unit] + headers)
        if not force and os.path.exists(obj) and os.path.getmtime(obj) > newest:
            continue
        cmd = [hipcc] + HIPCC_FLAGS + ["-c", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", obj, source]
        if verbose:
            print(" ".join(cmd), flush=True)
        running.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    said = [p.communicate()[0] for p in running]
    for p, out in zip(running, said):
        if p.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + out)
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objects, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("linking failed:\n" + r.stdout)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
