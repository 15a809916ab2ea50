"""Build libsrm.so (the HIP library behind include/srm.h) for gfx950 with hipcc."""
from __future__ import annotations

import glob
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libsrm.so")
# (srm.hip first: its code object is the first in the library)
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("srm.hip", "ops.hip")]
HEADERS = sorted(glob.glob(os.path.join(HERE, "csrc", "*.hpp"))) + [os.path.join(ROOT, "include", "srm.h")]


def build_lib(verbose: bool = False) -> str:
    """Compile unconditionally; returns the path of the shared library."""
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             "-I" + os.path.join(ROOT, "include"),
             # packed-fp32 VALU forms are kept off for every kernel of this library
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             # the first arguments of a kernel arrive in scalar registers instead of by a load of their own, the first trip to
             # memory of every launch (steps of few samples, chains of launches of 3 to 5 us: 2 to 5 % shorter)
             "-mllvm", "-amdgpu-kernarg-preload-count=16"]
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        jobs = [subprocess.Popen(["hipcc", *flags, "-c", src, "-o", obj], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
                for src, obj in zip(SOURCES, objects)]
        for job in jobs:                                   # (every compiler has ended when the first error is raised)
            job.out = job.communicate()
        link = None
        if not any(job.returncode for job in jobs):
            link = subprocess.run(["hipcc", "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", LIB], capture_output=True, text=True)
    for job in jobs:
        if verbose or job.returncode:
            print(*job.out)
        if job.returncode:
            raise RuntimeError("hipcc failed:\n" + job.out[1])
    if link.returncode:
        raise RuntimeError("linking failed:\n" + link.stderr)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS + [os.path.abspath(__file__)])


if __name__ == "__main__":
    print(build_lib(verbose=True))
