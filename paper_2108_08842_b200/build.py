"""Builds libeden.so (the CUDA kernels and their C ABI) for sm_100a with nvcc, and _binding.so
(the Python side of the training calls) with g++, both in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libeden.so")
BINDING = os.path.join(HERE, "_binding.so")
SOURCES = ["eden.cu", "train.cu", "lloyd_max.cpp", "uniform_family.cpp"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _newest_source() -> float:
    newest = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for name in os.listdir(root):
            newest = max(newest, os.path.getmtime(os.path.join(root, name)))
    return newest


def _fresh(obj: str) -> bool:
    """Whether an object is newer than every file that the compiler read for it."""
    try:
        with open(obj + ".d") as f:
            read = f.read().replace("\\\n", " ").split(":", 1)[1].split()
        made = os.path.getmtime(obj)
        return all(os.path.getmtime(p) <= made for p in read + [os.path.abspath(__file__)])
    except (OSError, IndexError):
        return False


def built_for() -> str:
    """What the extension depends on besides its sources: it holds this, and is only loaded by the same."""
    import torch

    return "torch %s, python %d.%d" % ((torch.__version__,) + sys.version_info[:2])


def _fresh_binding() -> bool:
    with open(BINDING, "rb") as f:
        if built_for().encode() not in f.read():
            return False
    own = [os.path.join(CSRC, "binding.cpp"), os.path.join(os.path.dirname(HERE), "include", "eden.h"), os.path.abspath(__file__)]
    return all(os.path.getmtime(p) <= os.path.getmtime(BINDING) for p in own)


def _binding_command(out: str) -> list:
    import sysconfig

    import torch

    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    libs = os.path.join(root, "lib")
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", '-DEDEN_BUILT_FOR="%s"' % built_for(), "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)] +
            ["-isystem" + i for i in includes] + ["-o", out,
            os.path.join(CSRC, "binding.cpp"), "-L" + libs, "-Wl,-rpath," + libs, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"])


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and all(os.path.exists(p) and os.path.getmtime(p) >= _newest_source() for p in (LIB, BINDING)) and _fresh_binding():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    mark = ".tmp.%d" % os.getpid()
    objects = [os.path.join(OBJ, s + ".o") for s in SOURCES]
    running = []
    for source, obj in zip(SOURCES, objects):           # one compiler per source, side by side
        if force or not _fresh(obj):
            cmd = [nvcc] + NVCC_FLAGS + ["-c", "-MMD", "-MF", obj + ".d", "-o", obj + mark, os.path.join(CSRC, source)]
            running.append((obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    if force or not os.path.exists(BINDING) or not _fresh_binding():
        running.append((BINDING, subprocess.Popen(_binding_command(BINDING + mark), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for made, p in running:
        out, _ = p.communicate()
        if verbose or p.returncode:
            sys.stderr.write(out)
        if p.returncode:
            failed.append(made)
        else:
            os.replace(made + mark, made)
    if any(made != BINDING for made in failed):
        raise RuntimeError("nvcc failed building libeden.so")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB + mark] + objects
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed linking libeden.so")
    os.replace(LIB + mark, LIB)
    if failed:
        if os.path.exists(BINDING):                     # made for what was there before
            os.remove(BINDING)
        raise RuntimeError("g++ failed building _binding.so, which the training calls need; libeden.so is built")
    os.utime(BINDING)
    return LIB


def main():
    print(build(force=True, verbose=True))


if __name__ == "__main__":
    main()
