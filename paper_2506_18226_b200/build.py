"""Builds, in-tree: libadsa.so (sm_100a) with nvcc, which knows nothing of torch; and adsa_marshal.so with g++, the part of the
Python binding that reads torch tensors in C++ (plain compiler calls, no torch extension machinery)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libadsa.so")
SOURCES = ["adsa_api.cu", "adsa_pool.cu", "adsa_score_select.cu", "adsa_attn.cu", "adsa_step.cu", "adsa_pstep.cu", "adsa_wstep.cu", "adsa_prefill.cu", "adsa_attn_static.cu", "adsa_shell.cu",
           "adsa_rotary.cu", "adsa_residual.cu", "adsa_prefix_attn.cu", "adsa_prefix_wide.cu", "adsa_prompt_attn.cu", "adsa_prompt_tile.cu", "adsa_prompt_few.cu", "adsa_sample.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]


MARSHAL = os.path.join(_HERE, "adsa_marshal.so")
MARSHAL_SOURCE = os.path.join(CSRC, "adsa_marshal.cpp")
HEADER = os.path.join(_HERE, "..", "include", "adsa.h")


def _stale(target: str, deps: list) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _built_against() -> bytes:
    """What the running interpreter's module says of itself (in the file, so that it can be asked without loading it)."""
    import re
    import sys

    import torch
    release = re.match(r"\d+\.\d+\.\d+", torch.__version__).group()
    return b"adsa_marshal built against torch %s, Python %d.%d;" % (release.encode(), *sys.version_info[:2])


def _foreign(path: str) -> bool:
    """Built against another torch or Python than the running one: it may not load, or read tensors wrongly."""
    with open(path, "rb") as f:
        return _built_against() not in f.read()


def build_marshal(force: bool = False) -> str:
    """Compile the tensor-reading half of the binding against the running torch."""
    if not force and not _stale(MARSHAL, [MARSHAL_SOURCE, HEADER]) and not _foreign(MARSHAL):
        return MARSHAL
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    include = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    libs = os.path.join(base, "lib")
    tmp = MARSHAL + f".tmp{os.getpid()}"
    # the system's g++, whatever CXX says: it links the shared C++ library that torch runs on, so that exceptions cross
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[f"-I{i}" for i in include], MARSHAL_SOURCE,
                           "-o", tmp, f"-L{libs}", f"-Wl,-rpath,{libs}", "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"])
    os.replace(tmp, MARSHAL)
    if _foreign(MARSHAL):
        raise ImportError(f"{MARSHAL}: the headers of this torch are another version's than {_built_against().decode()}")
    return MARSHAL


def build_lib(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu of the library for sm_100a and link libadsa.so next to this file."""
    if not force and not _stale(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [HEADER]):
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    # --threads: the sources are independent translation units, compiled side by side
    cmd = [nvcc, "--threads", str(min(len(SOURCES), os.cpu_count() or 1)), *NVCC_FLAGS, "-shared", "-o", tmp,
           *[os.path.join(CSRC, s) for s in SOURCES]]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build_lib(force=True, verbose="-v" in sys.argv))
    print(build_marshal(force=True))
