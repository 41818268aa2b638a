"""Builds libaugtree.so in-tree with hipcc for gfx950.

    python -m paper_2609_33133_amd.build [-v]

Every HIP source under csrc/ is compiled for --offload-arch=gfx950 (packed
fp32 instructions disabled), the host library as plain C++17, and all of it
linked into paper_2609_33133_amd/libaugtree.so. Always recompiles.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libaugtree.so")
BUILD = os.path.join(PKG, "_build")
ARCH = "gfx950"

COMMON = ["-O3", "-std=c++17", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I/opt/rocm/include"]
HIP_FLAGS = ["--offload-arch=" + ARCH, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-fno-honor-nans",
             "-ffp-contract=fast"]
# The linear-attention layer and the paged cache state how far a NaN or an
# infinity reaches, so their kernels are compiled with NaN honoured (ten of the
# 25000 lines of the linear layer's largest source differ, a paged attention
# kernel has 13 instructions more in 4200, and the times are the same).
NAN_SOURCES = ("linear", "head_norm", "paged", "attn_paged")
# The attention kernels are scheduled by the backend's instruction-level
# parallelism strategy (the dK/dV kernel runs ~1 % faster than with the
# default occupancy-driven one, the other two slightly faster; no spills);
# the bandwidth-bound merge and reduce kernels keep the default. The output and
# gradient kernels of linear attention gain 3-4 % from it.
ATTN_FLAGS = ["-mllvm", "-amdgpu-sched-strategy=max-ilp"]


def hip_flags(src: str):
    name = os.path.basename(src)
    flags = [f for f in HIP_FLAGS if f != "-fno-honor-nans" or not name.startswith(NAN_SOURCES)]
    return flags + (ATTN_FLAGS if name.startswith(("attn_", "linear.")) else [])


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("build failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    return r.stderr


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    cc = hipcc()
    jobs = []
    for src in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        jobs.append(([cc, "-x", "hip", *hip_flags(src), *COMMON, "-c", src, "-o", obj], obj))
    for src in sorted(glob.glob(os.path.join(CSRC, "*.cpp"))):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        jobs.append(([cc, "-x", "c++", "-D__HIP_PLATFORM_AMD__", *COMMON, "-c", src, "-o", obj], obj))
    with cf.ThreadPoolExecutor(max_workers=min(8, len(jobs))) as ex:
        list(ex.map(lambda j: _run(j[0], verbose), jobs))
    tmp = OUT + ".tmp"
    _run([cc, "--offload-arch=" + ARCH, "-shared", "-fPIC", "-o", tmp, *[o for _, o in jobs]], verbose)
    _check_kernel_stubs(tmp)
    os.replace(tmp, OUT)
    return OUT


def _check_kernel_stubs(lib: str) -> None:
    """Every kernel launch stub must be defined in the library: an undefined one
    would only fail when the library is loaded."""
    nm = shutil.which("nm") or "/usr/bin/nm"
    r = subprocess.run([nm, "-D", "--undefined-only", lib], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("nm failed on " + lib + ":\n" + r.stderr)
    missing = [ln.split()[-1] for ln in r.stdout.splitlines() if "__device_stub__" in ln]
    if missing:
        os.remove(lib)
        raise RuntimeError("kernel launch stubs missing from the library: " + ", ".join(missing))


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
