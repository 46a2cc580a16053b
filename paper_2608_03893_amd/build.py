"""Build libkvx.so (HIP for gfx950) and the binding's compiled part, _kvx_bind.so (host
C++), in the package directory.

Run ``python -m paper_2608_03893_amd.build``.  Every call recompiles.
"""

from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import time

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libkvx.so")
BIND = os.path.join(PKG, "_kvx_bind.so")
SOURCES = ["kvx_api.hip", "kvx_kernels.hip", "kvx_map_bf16.hip", "kvx_map_sweep.hip",
           "kvx_map_ks.hip", "kvx_map_ks_raw.hip", "kvx_map_tile.hip", "kvx_map_short.hip",
           "kvx_map_ks2.hip", "kvx_map_ks2_raw.hip", "kvx_xhead.hip", "kvx_noalloc.hip",
           "kvx_fit.hip", "kvx_mlp.hip", "kvx_serve.hip", "kvx_pages.hip", "kvx_store8.hip",
           "kvx_attend8.hip", "kvx_attend8_rows.hip"]

HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 VALU instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def hipcc() -> str:
    return os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def bind_command(out: str) -> list:
    """Compiles kvx_bind.cpp against the installed torch, which a process that imports the
    module has loaded."""
    import torch
    at = os.path.dirname(torch.__file__)
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
            "-isystem", os.path.join(at, "include"),
            "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
            "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "kvx_bind.cpp"),
            "-L", os.path.join(at, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python", "-o", out]


def build(verbose: bool = False) -> str:
    """Compile every source, link libkvx.so and the binding's compiled part; returns the
    library path.  libkvx.so needs hipcc alone: where the binding's part, which needs torch
    and a host compiler, cannot be built, it is linked all the same before the error."""
    t0 = time.time()
    objs = []
    procs = []
    bind = "kvx_bind.cpp"
    bind_failed = None
    try:
        cmd = bind_command(BIND + ".tmp")
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True), bind))
    except (ImportError, OSError) as e:      # no torch, no compiler
        bind_failed = str(e)
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [hipcc(), *HIP_FLAGS, "-I", INCLUDE, "-I", CSRC, "-c",
               os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((subprocess.Popen(cmd, stdout=subprocess.PIPE,
                                       stderr=subprocess.STDOUT, text=True), src))
        objs.append(obj)
    failed = []
    for p, src in procs:
        out, _ = p.communicate()
        # the host pass does not know the device-only feature flag: harmless
        lines = [ln for ln in out.splitlines()
                 if "packed-fp32-ops" not in ln]
        if lines and (verbose or p.returncode):
            print("\n".join(lines), file=sys.stderr)
        if p.returncode and src == bind:
            bind_failed = f"exit status {p.returncode}"
        elif p.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError(f"compilation failed for {failed}")
    tmp = LIB + ".tmp"
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    for o in objs:
        os.remove(o)
    if bind_failed is not None:
        if os.path.exists(BIND):      # an earlier library's
            os.remove(BIND)
        raise RuntimeError(f"compilation failed for {bind}: {bind_failed} ({LIB} is built)")
    os.replace(BIND + ".tmp", BIND)
    if verbose:
        print(f"built {LIB} in {time.time() - t0:.1f}s", flush=True)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
