"""Builds libvscan.so (sm_100a) in-tree with nvcc, and with the host compiler the module _calls.so that marshals the
arguments of the calls a decode step makes.  No torch types cross the library's boundary, so it is a plain shared object
loaded with ctypes; only _calls.so is built against torch."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB_PATH = os.path.join(HERE, "libvscan.so")

CALLS_PATH = os.path.join(HERE, "_calls.so")

STAMP_PATH = LIB_PATH + ".digest"

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=default", "-cudart", "static"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC)) + [os.path.join(INCLUDE, "vscan.h")]


def source_digest() -> str:
    """Digest of everything the library is built from (file names and contents, build flags)."""
    h = hashlib.sha256(" ".join(NVCC_FLAGS).encode())
    for path in _deps():
        h.update(os.path.basename(path).encode())
        with open(path, "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def _stale() -> bool:
    """True when libvscan.so or _calls.so is missing or was built from other sources than the ones on disk.  The
    digest recorded next to the library decides, not file times (a copied tree has arbitrary ones)."""
    if not os.path.exists(LIB_PATH) or not os.path.exists(CALLS_PATH) or not os.path.exists(STAMP_PATH):
        return True
    with open(STAMP_PATH) as f:
        return f.read().strip() != source_digest()


def have_nvcc() -> bool:
    return os.path.exists(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")


def _calls_command():
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"))
    dirs = [INCLUDE, *cpp_extension.include_paths(), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return (["g++", "-shared", "-fPIC", "-O2", "-std=c++17", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
            + [f"-I{d}" for d in dirs] + [os.path.join(CSRC, "calls.cpp"), "-o", CALLS_PATH, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into one shared library next to this file, and calls.cpp into the module beside it."""
    if not force and not _stale():
        return LIB_PATH
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        raise RuntimeError("nvcc not found: libvscan.so cannot be built")
    digest = source_digest()
    cmd = [nvcc, "-shared", "-o", LIB_PATH, "-I", INCLUDE, "-I", CSRC] + NVCC_FLAGS
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += sources()
    calls = subprocess.Popen(_calls_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    said = calls.communicate()[0]
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if calls.returncode != 0:
        raise RuntimeError("g++ failed:\n" + said)
    with open(STAMP_PATH, "w") as f:
        f.write(digest + "\n")
    if verbose:
        sys.stderr.write(res.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
