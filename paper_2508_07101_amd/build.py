"""Builds libcusa.so (gfx950) in-tree from csrc/ with hipcc."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libcusa.so")
SOURCES = [os.path.join(CSRC, f) for f in ("cusa.hip", "tree.hip", "beam.hip", "build_id.hip")]
HEADERS = [os.path.join(CSRC, f) for f in ("attn_parts.hpp", "attn_plan.hpp", "beam_attn.hpp", "beam_kernels.hpp", "beam_plan.hpp", "cache_view.hpp", "call_tag.hpp", "cusa_kernels.hpp", "host.hpp", "plan_scan.hpp", "tree_kernels.hpp",
                                           "tree_plan.hpp")]
HEADERS.append(os.path.join(os.path.dirname(_HERE), "include", "cusa.h"))

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-FP32 forms are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the leading kernel arguments arrive in SGPRs with the wave instead of through a first load
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: libcusa cannot be built")
    return exe


def source_id() -> str:
    """Digest of everything the library is compiled from (sources, headers, flags); the library
    carries the digest it was built from (cusa_build_id), which is how a stale binary is told."""
    h = hashlib.sha256()
    for f in SOURCES + HEADERS:
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(HIPCC_FLAGS).encode())
    return h.hexdigest()[:16]


def build_lib(force: bool = True, extra_flags=()) -> str:
    """Compile the library, its sources side by side; with force=False only when it is missing."""
    if not force and os.path.exists(LIB):
        return LIB
    tmp = LIB + f".tmp{os.getpid()}"
    objects = [f"{tmp}.{i}.o" for i in range(len(SOURCES))]
    flags = [*HIPCC_FLAGS, f'-DCUSA_BUILD_ID="{source_id()}"', *extra_flags]
    try:
        jobs = [subprocess.Popen([hipcc(), *flags, "-c", "-o", obj, src]) for src, obj in zip(SOURCES, objects)]
        for src, status in [(src, job.wait()) for src, job in zip(SOURCES, jobs)]:
            if status:
                raise subprocess.CalledProcessError(status, f"hipcc -c {src}")
        subprocess.check_call([hipcc(), "--offload-arch=gfx950", "-shared", *extra_flags, "-o", tmp, *objects])
        os.replace(tmp, LIB)
    finally:
        for f in objects + [tmp]:
            if os.path.exists(f):
                os.remove(f)
    return LIB


if __name__ == "__main__":
    print(build_lib(True))
