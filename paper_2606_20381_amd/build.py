"""Build libufp4.so (gfx950) and the binding's host module in-tree with hipcc.

Usage: python -m paper_2606_20381_amd.build [--verbose]

Every translation unit is compiled for gfx950 only, without packed-fp32 instructions, with fp contraction
off (the quantizer's arithmetic must round exactly as written) and denormals preserved (no fast-math).
"""

from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libufp4.so")
HOST = os.path.join(PKG, "_host.so")  # a Python module: the host side of short calls, on torch's C++ interface and libufp4.so
INCLUDE = os.path.join(os.path.dirname(PKG), "include")

SOURCES = ["ufp4_quant.hip", "ufp4_gemm.hip", "ufp4_gemm_mx.hip", "ufp4_mxfp4.hip", "ufp4_gemm_mxfp4.hip",
           "ufp4_linear_mxfp4.hip", "ufp4_norm.hip", "ufp4_moe.hip", "ufp4_gemm_bf16.hip", "ufp4_ckpt8.hip", "ufp4_api.cpp",
           "ufp4_api_layer.cpp", "ufp4_api_bf16.cpp"]

ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
    "-Wno-unused-function",
]
# MFMA results in VGPRs: the GEMM epilogue reads them with plain VALU FMAs (no AGPR copies). Not the microscaled 4-bit GEMM,
# whose largest tile holds 128 results a lane and two sets of operands: with the results in AGPRs nothing is spilled.
VGPR_FORM = ["-mllvm", "-amdgpu-mfma-vgpr-form"]
AGPR_SOURCES = ("ufp4_gemm_mxfp4.hip",)


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    exe = shutil.which("hipcc") or os.path.join(rocm, "bin", "hipcc")
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found")
    return exe


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"command failed ({r.returncode}): {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if verbose and r.stderr.strip():
        print(r.stderr, file=sys.stderr)
    return r


def _host_object(cc: str) -> tuple[list, str, str] | None:
    """(command that compiles the host module, its object file, torch's library folder), None where there is no torch."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    torch = os.path.dirname(spec.origin)
    inc = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include")]
    obj = os.path.join(BUILD, "ufp4_host.o")
    return ([cc, "-x", "c++", "-std=c++17", "-O2", "-fPIC", "-Wall", "-Wno-unused-function", f"-I{INCLUDE}",
             f"-I{sysconfig.get_paths()['include']}", *(x for i in inc for x in ("-isystem", i)), "-c",
             os.path.join(CSRC, "ufp4_host.cpp"), "-o", obj], obj, os.path.join(torch, "lib"))


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library and the host module; always rebuilds. Returns the library path. The library needs
    no torch: without one (or where the host module does not compile, which raises) it is built all the same."""
    os.makedirs(BUILD, exist_ok=True)
    cc = hipcc()
    objs = []
    cmds = []
    for src in SOURCES:
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        lang = ["-x", "hip"] if src.endswith(".cpp") else []
        form = [] if src in AGPR_SOURCES else VGPR_FORM
        cmds.append([cc, *FLAGS, *form, f"-I{INCLUDE}", *lang, "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    host = _host_object(cc)
    with ThreadPoolExecutor(max_workers=len(cmds) + 1) as ex:
        host_done = ex.submit(_run, host[0], verbose) if host else None
        list(ex.map(lambda c: _run(c, verbose), cmds))
    tmp = LIB + ".tmp"
    _run([cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs], verbose)
    os.replace(tmp, LIB)
    if host is None:
        print("no torch: the binding's host module is not built", file=sys.stderr)
        return LIB
    host_done.result()
    _, host_obj, torch_lib = host
    tmp = HOST + ".tmp"  # torch's libraries are loaded by the time the module is
    _run([cc, "-shared", "-fPIC", "-o", tmp, host_obj, f"-L{PKG}", "-l:libufp4.so", "-Wl,-rpath,$ORIGIN", f"-L{torch_lib}",
          "-ltorch_python", "-ltorch_cpu", "-lc10"], verbose)
    os.replace(tmp, HOST)
    return LIB


if __name__ == "__main__":
    print(build(verbose="--verbose" in sys.argv))
