"""Build the C-ABI library liblstm_approx.so in-tree with nvcc for sm_103a,
and the module _torch_ops that passes torch tensors to its operators.

Each translation unit is compiled in parallel, then linked into one shared
library and one module next to this file.  Objects go to ``_build/``
(git-ignored).
"""
from __future__ import annotations

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "liblstm_approx.so")
MODULE = os.path.join(HERE, "_torch_ops.so")
MODULE_FOR = os.path.join(BUILD, "torch_ops.torch")  # what the module was compiled for, see _torch_abi
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
                     "--expt-relaxed-constexpr", "-I" + INCLUDE]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]


def up_to_date() -> bool:
    """Whether the library, and where there is a torch the module, are newer than every source (and for that torch)."""
    made = [LIB] + ([MODULE] if _torch_dir() else [])
    if not all(os.path.exists(p) for p in made):
        return False
    if _torch_dir() and not (os.path.exists(MODULE_FOR) and open(MODULE_FOR).read() == _torch_abi()):
        return False
    t = min(os.path.getmtime(p) for p in made)
    return all(os.path.getmtime(p) <= t for p in _deps())


def _run(cmd, what: str, verbose: bool = False):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what}:\n{r.stdout}\n{r.stderr}")
    if verbose and (r.stdout or r.stderr):
        sys.stderr.write(r.stdout + r.stderr)


def _torch_dir():
    """Where torch is; None without one (the library needs none, the module is for it alone)."""
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec else None


def _torch_abi() -> str:
    """The torch and the Python that the module is for: with another one of either it may not load."""
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        return f"{f.read()}\n{sysconfig.get_config_var('SOABI')}\n"


def _compile_module() -> str:
    torch, obj = _torch_dir(), os.path.join(BUILD, "torch_ops.o")
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    include = [INCLUDE, sysconfig.get_paths()["include"], os.path.join(torch, "include"),
               os.path.join(torch, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", *("-I" + d for d in include), "-c",
          os.path.join(CSRC, "torch_ops.cpp"), "-o", obj], "g++ failed for torch_ops.cpp")
    return obj


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile every .cu under csrc/, link liblstm_approx.so and, where there is a torch, the operators' module;
    returns the library's path."""
    if not force and up_to_date():
        return LIB
    nvcc = _nvcc()
    os.makedirs(BUILD, exist_ok=True)
    srcs = sources()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj]
        _run(cmd, f"nvcc failed for {src}", verbose)
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as ex:
        module = ex.submit(_compile_module) if _torch_dir() else None
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB + ".tmp"
    _run([nvcc, *ARCH, "-shared", "-o", tmp, *objs], "link failed")
    os.replace(tmp, LIB)
    if module is None:
        return LIB
    tmp = MODULE + ".tmp"
    _run(["g++", "-shared", "-o", tmp, module.result(), "-L" + os.path.join(_torch_dir(), "lib"), "-ltorch", "-ltorch_python",
          "-lc10", "-lc10_cuda", "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"], "module link failed")
    os.replace(tmp, MODULE)
    with open(MODULE_FOR, "w") as f:
        f.write(_torch_abi())
    return LIB


if __name__ == "__main__":
    v = "-v" in sys.argv
    print(build(force=True, verbose=v, extra_flags=(["-Xptxas", "-v"] if v else [])))
