"""Builds libckv.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libckv.so")
MARSHAL = os.path.join(HERE, "_marshal.so")        # the binding's argument checks (a Python extension)
MARSHAL_FOR = os.path.join(HERE, "_build", "marshal_for")   # the Python and torch that it was built for

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--expt-relaxed-constexpr",
]


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build_lib(force: bool = False, verbose: bool = False) -> str:
    build_marshal(force)
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    procs = []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for src in sources():
        obj = os.path.join(HERE, "_build", os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((cmd, subprocess.Popen(cmd)))
        objs.append(obj)
    for cmd, p in procs:
        if p.wait() != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    link = [nvcc, "-shared", "-o", LIB, *objs, "-gencode", "arch=compute_100a,code=sm_100a"]
    subprocess.check_call(link)
    return LIB


def built_for() -> str:
    from importlib.metadata import version
    return f"{sys.version}\ntorch {version('torch')}\n"


def marshal_stale() -> bool:
    """Older than its source, or built for another Python or torch (or nobody knows for which)."""
    if not (os.path.exists(MARSHAL) and os.path.exists(MARSHAL_FOR)):
        return True
    with open(MARSHAL_FOR) as f:
        return f.read() != built_for() or os.path.getmtime(MARSHAL) < os.path.getmtime(os.path.join(CSRC, "marshal.cpp"))


def build_marshal(force: bool = False) -> str:
    src = os.path.join(CSRC, "marshal.cpp")
    if not force and not marshal_stale():
        return MARSHAL
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    out = MARSHAL[:-3] + f".{os.getpid()}.so"          # another process may be loading the one there is
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", *[a for i in inc for a in ("-isystem", i)],
                           src, "-o", out, "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])
    os.replace(out, MARSHAL)
    os.makedirs(os.path.dirname(MARSHAL_FOR), exist_ok=True)
    with open(MARSHAL_FOR, "w") as f:
        f.write(built_for())
    return MARSHAL


if __name__ == "__main__":
    print(build_lib(force="--force" in sys.argv, verbose="-v" in sys.argv))
