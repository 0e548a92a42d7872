"""Build ``libquasar.so`` (HIP for gfx950) in-tree with hipcc.

Flags that matter for results:
  -ffp-contract=off      no implicit a*b+c -> fma; every fma in the kernels is explicit
  (default) correctly rounded fp32 division and IEEE denormals (no -ffast-math)
  -Xclang -target-feature -Xclang -packed-fp32-ops
                         no packed-fp32 (v_pk_*_f32) instructions are generated
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libquasar.so")
SOURCES = ["api.hip", "int_kernel.hip", "int_cells_kernel.hip", "nvfp4_kernel.hip", "rubin_kernel.hip",
           "ops_api.hip", "norm_kernel.hip", "distill_kernel.hip", "linear_kernel.hip", "layer_norm_kernel.hip",
           "embed_kernel.hip", "checkpoint_kernel.hip", "weight_grad_kernel.hip"]
ARCH = "gfx950"
BINDING = os.path.join(HERE, "_ops_binding.so")  # the Python calls of ops.py, in C++

COMMON = ["-O3", "-std=c++17", f"--offload-arch={ARCH}", "-fPIC", "-ffp-contract=off",
          "-fno-fast-math", "-fno-gpu-rdc", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wall", "-Wno-unused-function", "-Wno-unknown-warning-option",
          f"-I{INCLUDE}", f"-I{CSRC}"]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc(), *COMMON, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def _build_binding(verbose: bool) -> str:
    """The host-only extension module of ops.py (torch's C++ API; its device work is libquasar.so's)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    obj = os.path.join(BUILD, "ops_binding.o")
    cxx = os.environ.get("CXX", "g++")
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-Wno-unknown-pragmas", "-Wno-attributes",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{INCLUDE}",
           *[f"-isystem{p}" for p in cpp_extension.include_paths()], f"-isystem{sysconfig.get_paths()['include']}",
           "-c", os.path.join(CSRC, "ops_binding.cpp"), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cxx} failed for ops_binding.cpp:\n{r.stderr}")
    return obj


def _link_binding(obj: str, verbose: bool) -> None:
    from torch.utils import cpp_extension
    tmp = BINDING + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-shared", "-o", tmp, obj, f"-L{HERE}", "-l:libquasar.so", "-Wl,-rpath,$ORIGIN",
           *[f"-L{p}" for p in cpp_extension.library_paths()], "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, BINDING)


def build(verbose: bool = False, extra_flags=()) -> str:
    """Compile every HIP source for gfx950 and link libquasar.so and the binding of its operators (always rebuilds)."""
    os.makedirs(BUILD, exist_ok=True)
    global COMMON
    if extra_flags:
        COMMON = COMMON + list(extra_flags)
    with ThreadPoolExecutor(len(SOURCES) + 1) as ex:
        binding = ex.submit(_build_binding, verbose)
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
        binding = binding.result()
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    _link_binding(binding, verbose)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
