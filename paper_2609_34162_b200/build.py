"""Builds libslidedp.so in-tree with nvcc for sm_100a (cross-compiles without a GPU).

Usage: python -m paper_2609_34162_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import re
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libslidedp.so")
MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")     # the binding's own part in C++, for this interpreter and torch
SOURCES = [os.path.join(CSRC, f) for f in ("common.cu", "context.cu", "update.cu", "stream.cu",
                                           "model.cu", "ipc.cu", "qk_norm_rope.cu", "distill.cu",
                                           "attention.cu", "attention_mma.cu", "embedding.cu",
                                           "block_norm.cu", "policy.cu", "clip.cu")]
DEPENDS = SOURCES + [os.path.join(CSRC, f) for f in ("kernels.cuh", "cast_kernel.cuh",
                                                     "device_utils.cuh", "types.h", "internal.h",
                                                     "ops_internal.h", "attention.h",
                                                     "attention_rows.cuh", "tcgen05.cuh",
                                                     "logit_rows.cuh", "rows.cuh")]
DEPENDS += [os.path.join(ROOT, "include", f) for f in ("slidedp.h", "slidedp_ops.h")]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def marshal_name() -> str:
    """The module's name: it is compiled against this torch's headers, and another torch must not load it."""
    import torch
    return "_marshal_torch_" + re.sub(r"\W", "_", torch.__version__)


def build_marshal(force: bool = False) -> str:
    name = marshal_name()
    path = os.path.join(PKG, name + sysconfig.get_config_var("EXT_SUFFIX"))
    if force or not os.path.exists(path) or os.path.getmtime(path) < os.path.getmtime(MARSHAL_SOURCE):
        import torch
        torch_dir = os.path.dirname(torch.__file__)
        tmp = path + ".tmp.%d" % os.getpid()
        include = [sysconfig.get_paths()["include"], os.path.join(torch_dir, "include"),
                   os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
                   os.path.join(os.path.dirname(os.path.dirname(nvcc())), "include")]
        subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
                        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", f"-DMARSHAL_NAME={name}"]
                       + [f"-I{d}" for d in include] + ["-o", tmp, MARSHAL_SOURCE, "-L" + os.path.join(torch_dir, "lib"),
                       "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"], check=True)
        os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    build_marshal(force)
    stale = (not os.path.exists(LIB)
             or os.path.getmtime(LIB) < max(os.path.getmtime(p) for p in DEPENDS))
    if force or stale:
        tmp = LIB + ".tmp.%d" % os.getpid()
        cmd = [nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3",
               "--threads", "0",
               "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
               "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", tmp] + SOURCES
        if verbose:
            cmd.insert(1, "-Xptxas"); cmd.insert(2, "-v")
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
