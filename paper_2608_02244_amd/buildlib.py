"""Build libfsched.so in-tree with hipcc for gfx950.

Every HIP translation unit under csrc/ is compiled in parallel, then linked
into one shared library next to this file; the binding of the step's operators
(csrc/bind) becomes an extension module beside it, compiled against torch (left out
where torch is not installed: the evaluation calls work on numpy arrays without it).
No CPU fallback is built.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import importlib.util
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libfsched.so")
BIND_SRC = os.path.join(CSRC, "bind", "step_bind.cpp")
BIND_LIB = os.path.join(HERE, "_step.so")
BUILD_DIR = os.path.join(HERE, "_build")

ARCH = "gfx950"
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Werror=inline-asm",  # clobbers that the compiler does not honour
          f"-I{INCLUDE}", f"-I{CSRC}"]
# Instruction scheduling strategies, chosen by measurement: the simulation
# kernels (csrc/sim_*.hip) by LLVM's iterative max-occupancy strategy, the
# re-scoring kernel by max-ILP (with the other's strategy each ran slower); the
# other sources keep the default.
SIM_FLAGS = ["-mllvm", "-amdgpu-sched-strategy=iterative-maxocc"]
DEC_FLAGS = ["-mllvm", "-amdgpu-sched-strategy=max-ilp"]


def _flags(src: str) -> list:
    name = os.path.basename(src)
    if name.startswith("sim_"):
        return SIM_FLAGS
    if name == "decompose.hip":
        return DEC_FLAGS
    return []


def _hipcc() -> str:
    h = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(h):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return h


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [_hipcc()] + COMMON + _flags(src) + lang + ["-c", src, "-o", obj]
    _run(cmd, "compile")
    return obj


def _run(cmd: list, what: str) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")


def _cxx() -> list:
    """A host C++ compiler: hipcc where there is no other."""
    found = shutil.which("g++") or shutil.which("c++")
    return [found] if found else [_hipcc()]


def _compile_bind() -> str:
    """Object file of the binding (host code only)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    obj = os.path.join(BUILD_DIR, "step_bind.o")
    inc = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], INCLUDE]
    _run(_cxx() + ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden",
                   f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] +
         [f"-I{p}" for p in inc] + ["-x", "c++", "-c", BIND_SRC, "-o", obj], "compile")
    return obj


def _link_bind(obj: str) -> None:
    """The extension module, which finds libfsched.so beside it (torch's libraries are
    loaded by the time it is imported)."""
    from torch.utils import cpp_extension
    lib = cpp_extension.library_paths()[0]
    tmp = BIND_LIB + ".tmp"
    _run(_cxx() + ["-shared", "-o", tmp, obj, f"-L{HERE}", "-lfsched", f"-L{lib}", "-lc10",
          "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"], "link")
    os.replace(tmp, BIND_LIB)


def build(jobs: int | None = None, verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))
    jobs = jobs or min(len(srcs), os.cpu_count() or 4, 16)
    with_bind = importlib.util.find_spec("torch") is not None
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        bind = ex.submit(_compile_bind) if with_bind else None
        objs = list(ex.map(_compile, srcs))
        bind_obj = bind.result() if with_bind else None
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    _run(cmd, "link")
    os.replace(tmp, LIB)
    if with_bind:
        _link_bind(bind_obj)
    else:
        if os.path.exists(BIND_LIB):
            os.remove(BIND_LIB)  # of an older libfsched.so
        print("torch is not installed: built without the step operators' binding")
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
