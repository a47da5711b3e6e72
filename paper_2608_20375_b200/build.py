"""Build libgraft.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a.

Every source becomes an object under _build/ (rebuilt when it or one of its headers is newer) and the objects are
linked into libgraft.so.  The binding's checks of tensors for calls of a few microseconds are host code against torch's and Python's headers, a module
of its own that nothing needs: where it does not compile, the library is there without it.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libgraft.so")
GRAFT_H = os.path.join("..", "..", "include", "graft.h")
ALL_HEADERS = ["common.cuh", "internal.h", "edge_score.cuh", "cosine.cuh", "saba.cuh", GRAFT_H]
# source -> headers it depends on
SOURCES = {
    "api.cu": ALL_HEADERS,
    "vocab_pass.cu": ALL_HEADERS + ["umma.cuh", "vocab_common.cuh", "vocab_rows.cuh"],
    "tdes.cu": ALL_HEADERS,
    "tree.cu": ALL_HEADERS,
    "tdes_train.cu": ["common.cuh", "internal.h", GRAFT_H],
    "saba_fit.cu": ["common.cuh", "internal.h", GRAFT_H],
    "cache.cu": ["common.cuh", "internal.h", "cache.cuh", GRAFT_H],
    "append.cu": ["common.cuh", "internal.h", "cache.cuh", GRAFT_H],
    "window_attn.cu": ["common.cuh", "internal.h", "cache.cuh", "umma.cuh", "attn.cuh", GRAFT_H],
    "tree_attn.cu": ["common.cuh", "internal.h", "cache.cuh", "umma.cuh", "attn.cuh", GRAFT_H],
    "verify.cu": ["common.cuh", "internal.h", "umma.cuh", GRAFT_H],
    "tables_mma.cu": ["common.cuh", "internal.h", "umma.cuh", GRAFT_H],
}
# no --use_fast_math: the fp64 pieces (log-sum-exp fold, SABA) and the fp32 divisions must stay IEEE
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _stale(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _obj(src: str) -> str:
    return os.path.join(OBJ, src.replace(".cu", ".o"))


def needs_build() -> bool:
    for src, hdrs in SOURCES.items():
        if _stale(_obj(src), [os.path.join(CSRC, src)] + [os.path.join(CSRC, h) for h in hdrs]):
            return True
    return _stale(LIB, [_obj(s) for s in SOURCES])


def _marshal_deps() -> list[str]:
    return [os.path.join(CSRC, "marshal.cpp"), os.path.join(CSRC, GRAFT_H)]


def marshal_path() -> str:
    """The compiled checks of this Python and this torch: where tensors keep what is read of them differs from one to another."""
    import torch
    return os.path.join(HERE, f"_marshal.torch-{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}")


def _marshal_command(out: str) -> list[str]:
    import torch
    at = os.path.dirname(torch.__file__)
    inc = [os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] +
            [f"-I{i}" for i in inc] + [os.path.join(CSRC, "marshal.cpp"), "-o", out, "-L" + os.path.join(at, "lib"), "-ltorch_python",
                                       "-ltorch_cpu", "-lc10"])


def build_marshal(force: bool = False) -> str | None:
    """The compiled checks, compiled if they are missing or stale; None, with a warning, where that fails."""
    path = marshal_path()
    if force or _stale(path, _marshal_deps()):
        part = f"{path}.{os.getpid()}"  # (whoever loads it meanwhile sees all of it or nothing)
        try:
            subprocess.run(_marshal_command(part), check=True, capture_output=True, text=True)
            os.replace(part, path)
        except (OSError, subprocess.CalledProcessError) as e:
            if os.path.exists(part):
                os.unlink(part)
            warnings.warn(f"the binding's compiled checks could not be built, calls check their arguments in Python: {e}\n{getattr(e, 'stderr', '') or ''}")
            return None
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    inc = ["-I", os.path.join(HERE, "..", "include")]
    cmds = []
    for src, hdrs in SOURCES.items():
        deps = [os.path.join(CSRC, src)] + [os.path.join(CSRC, h) for h in hdrs]
        if not (force or _stale(_obj(src), deps)):
            continue
        cmds.append([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + inc +
                    ["-c", os.path.join(CSRC, src), "-o", _obj(src)])
    procs = [subprocess.Popen(c) for c in cmds]  # the sources compile side by side
    build_marshal(force)
    failed = [c for c, pr in zip(cmds, procs) if pr.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])
    if force or _stale(LIB, [_obj(s) for s in SOURCES]):
        subprocess.check_call([nvcc, "-shared", "-o", LIB] + [_obj(s) for s in SOURCES] + ["-lcudart"])
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
