"""Compile the HIP library (csrc/*.hip -> libriver.so) for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC = os.path.join(HERE, "csrc", "river.hip")
# one object per source, river.hip's code object first in the library
SOURCES = [SRC, *(os.path.join(HERE, "csrc", s) for s in ("river_pages.hip", "river_prefix.hip", "river_step.hip"))]
DEPS = [*SOURCES, *(os.path.join(HERE, "csrc", h) for h in ("river_copies.h", "river_device.h", "river_prefill.h", "river_host.h", "river_pages.h",
                                                            "river_pages_host.h", "river_pool.h", "river_prefix.h", "river_step.h")),
        os.path.join(ROOT, "include", "river.h")]
LIB = os.path.join(HERE, "libriver.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # packed-fp32 instruction selection is switched off on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-parameter",
]


def is_stale() -> bool:
    return (not os.path.exists(LIB)
            or any(os.path.getmtime(LIB) < os.path.getmtime(d) for d in DEPS))


TRACE_LIB = os.path.join(HERE, "libriver_trace.so")


def build(force: bool = True, trace: bool = False) -> str:
    """trace=True builds the diagnostics variant (per-barrier device timestamps)."""
    out = TRACE_LIB if trace else LIB
    if not force and not trace and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [*HIPCC_FLAGS, *(["-DRIVER_TRACE"] if trace else []), "-I", os.path.join(ROOT, "include")]
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    objects = [os.path.join(HERE, "_build", os.path.basename(s) + (".trace.o" if trace else ".o")) for s in SOURCES]
    running = [subprocess.Popen([hipcc, *flags, "-c", "-o", o, s]) for s, o in zip(SOURCES, objects)]
    codes = [p.wait() for p in running]
    for s, rc in zip(SOURCES, codes):
        if rc:
            raise subprocess.CalledProcessError(rc, f"{hipcc} -c {s}")
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", out, *objects], check=True)
    return out


if __name__ == "__main__":
    print(build())
