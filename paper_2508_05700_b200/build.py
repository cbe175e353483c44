"""Builds libmfet.so (the C-ABI CUDA library) in-tree for sm_100a with nvcc."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmfet.so")
LIB_CHECKED = os.path.join(HERE, "libmfet_checked.so")  # the same library with -DMFET_CHECKED (see common.cuh)
FASTCALL = os.path.join(HERE, "_fastcall" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))  # Python entry of the hot calls
SOURCES = ["api.cu", "bag.cu", "hash_fill.cu", "dedup.cu", "hostpath.cu", "backward.cu", "rows.cu",
           "gradclip.cu", "mx4.cu", "norm.cu", "gated.cu", "ortho.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O3", "-lineinfo",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--fmad=true"]


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def build_fastcall(force: bool = False) -> str | None:
    """The binding's extension (host code: csrc/fastcall.c). Where it cannot be built (no compiler or headers for this Python) there is none:
    the binding then makes its calls through ctypes."""
    src = os.path.join(CSRC, "fastcall.c")
    deps = [src, os.path.join(HERE, "..", "include", "mfet.h")]
    if force or not os.path.exists(FASTCALL) or os.path.getmtime(FASTCALL) < _newest(deps):
        tmp = FASTCALL + ".tmp.%d" % os.getpid()
        try:
            subprocess.check_call([os.environ.get("CC", "gcc"), "-O2", "-fPIC", "-shared", "-Wall", "-I", sysconfig.get_paths()["include"],
                                   src, "-o", tmp])
        except (OSError, subprocess.CalledProcessError) as e:
            sys.stderr.write("no extension for the binding, its calls go through ctypes: %s\n" % e)
            if os.path.exists(FASTCALL):  # of an older source
                os.remove(FASTCALL)
            return None
        os.replace(tmp, FASTCALL)
    return FASTCALL


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Builds (if out of date) and returns the library; checked=True: the bounds-checked build, in
    which the kernels test the indices of their loads and stores and report a violation through MFET_DEV_BOUNDS (what the tensor-map
    copies of the MXFP4 product reach is clipped by the map)."""
    build_fastcall(force)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    deps = srcs + [os.path.join(CSRC, "common.cuh"), os.path.join(CSRC, "dedup_layout.cuh"), os.path.join(CSRC, "lowbit.cuh"),
                   os.path.join(CSRC, "tensor.cuh"), os.path.join(CSRC, "gemm16.cuh"),
                   os.path.join(HERE, "..", "include", "mfet.h")]
    lib = LIB_CHECKED if checked else LIB
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= _newest(deps):
        return lib
    objs = []
    procs = []
    for s in srcs:
        o = os.path.join(CSRC, os.path.basename(s)[:-3] + (".checked.o" if checked else ".o"))
        cmd = [nvcc] + NVCC_FLAGS + (["-DMFET_CHECKED"] if checked else []) + (["-Xptxas", "-v"] if verbose else []) + \
            ["-c", s, "-o", o]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(o)
    for cmd, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    tmp = lib + ".tmp.%d" % os.getpid()
    subprocess.check_call([nvcc, "-shared", "-o", tmp] + objs + ["-lcudart"])
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
