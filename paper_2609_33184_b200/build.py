"""Build libspecstream.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libspecstream.so")
MARSHAL = os.path.join(PKG, "_marshal.so")   # the binding's argument marshalling (csrc/marshal.cpp)
SOURCES = ["api.cu", "chunk_simt.cu", "chunk_tc.cu", "chunk_tc_keys.cu", "local_finalize.cu", "stream_round.cu", "static_round.cu", "tier.cu", "width.cu", "cohort.cu", "probe.cu",
           "kv8_copy.cu", "kv8_attn_simt.cu", "kv8_attn_tc.cu", "kv8_join.cu", "rope.cu", "window_attn_tc.cu"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths.append(os.path.join(ROOT, "include", "specstream.h"))
    return max(os.path.getmtime(p) for p in paths)


def _run(cmd) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(os.path.basename(cmd[0]) + " failed:\n" + res.stdout + res.stderr)
    return res.stderr


def build_marshal() -> None:
    """The extension module that checks tensors and calls the library, linked to it and to torch."""
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    _run([os.environ.get("CXX", "g++"), "-shared", "-fPIC", "-O2", "-std=c++17", "-o", MARSHAL,
          os.path.join(CSRC, "marshal.cpp"), "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
          "-I", os.path.join(torch, "include"), "-I", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
          "-L", PKG, "-l:libspecstream.so", "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
          "-Wl,-rpath,$ORIGIN"])


def build(force: bool = False, verbose: bool = False) -> str:
    newest = _newest_source_mtime()
    if not force and all(os.path.exists(f) and os.path.getmtime(f) >= newest for f in (LIB, MARSHAL)):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-shared", "-o", LIB, "-std=c++17", "-O3", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-cudart", "static"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    said = _run(cmd)
    build_marshal()
    if verbose:
        print(said)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
