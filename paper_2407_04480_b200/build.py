"""Compile the CUDA library in-tree with nvcc for sm_100a.

    python -m paper_2407_04480_b200.build [--force] [--verbose]

Produces paper_2407_04480_b200/libloco_b200.so, libloco_layer_b200.so (the operators of a
decoder layer, include/loco_layer.h) and _layer_binding.so (the native half of layer.py, the only
part that needs torch's headers) next to this file.  nvcc cross-compiles without a GPU, so
this runs anywhere the CUDA toolkit is installed.  The kernel templates are instantiated in
several object files (see csrc/loco_dispatch.h) that are compiled in parallel and linked into
one shared library each; the objects live in a temporary directory.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libloco_b200.so")
DEPS = [os.path.join(CSRC, f) for f in ("loco_api.cu", "loco_send_tu.cu", "loco_reduce_tu.cu", "loco_kernels.cuh",
                                        "loco_dispatch.h")] + [os.path.join(os.path.dirname(HERE), "include", "loco.h")]
LAYER_LIB = os.path.join(HERE, "libloco_layer_b200.so")
LAYER_SOURCES = ("layer_rotary.cu", "layer_router.cu", "layer_attention.cu", "layer_attention_api.cu", "layer_norm.cu", "layer_experts.cu",
                 "layer_product.cu", "layer_gradient.cu")
LAYER_DEPS = [os.path.join(CSRC, f) for f in LAYER_SOURCES + ("layer_common.h", "layer_attention.h", "layer_maps.h", "layer_tc.cuh")] + [
    os.path.join(os.path.dirname(HERE), "include", f) for f in ("loco.h", "loco_layer.h")]
BINDING = os.path.join(HERE, "_layer_binding.so")
BINDING_DEPS = [os.path.join(CSRC, "layer_binding.cpp")] + [os.path.join(os.path.dirname(HERE), "include", f) for f in ("loco.h", "loco_layer.h")]

NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC"]


def units():
    """(object name, source, extra defines) of every translation unit."""
    out = [("api", "loco_api.cu", [])]
    for g in (0, 1):
        for s in (0, 1, 2, 3):
            out.append(("send_g%d_s%d" % (g, s), "loco_send_tu.cu", ["-DLOCO_TU_GRAD=%d" % g, "-DLOCO_TU_STATE=%d" % s]))
    for o in (0, 1):
        for a in (0, 1):
            out.append(("reduce_o%d_a%d" % (o, a), "loco_reduce_tu.cu", ["-DLOCO_TU_OUT=%d" % o, "-DLOCO_TU_ADAM=%d" % a]))
    return out


def nvcc_path() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found: the LoCo CUDA library cannot be built")
    return p


def stale(lib: str = LIB, deps=DEPS) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(d) > t for d in deps)


def binding_for() -> str:
    """What the binding is built for: it loads with this torch and interpreter only."""
    from importlib.metadata import version
    return "built for torch %s, python %d.%d" % (version("torch"), *sys.version_info[:2])


def stale_binding() -> bool:
    if stale(BINDING, BINDING_DEPS):
        return True
    with open(BINDING, "rb") as f:                       # its docstring
        return binding_for().encode() not in f.read()


def build_binding() -> None:
    """The Python module that marshals layer.py's calls, linked against the layer library and torch."""
    import torch
    home, cuda = os.path.dirname(torch.__file__), os.path.dirname(os.path.dirname(nvcc_path()))
    tmp = BINDING + ".tmp.%d" % os.getpid()
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I" + os.path.join(home, "include"),
                           "-I" + os.path.join(home, "include", "torch", "csrc", "api", "include"), "-I" + os.path.join(cuda, "include"),
                           "-I" + sysconfig.get_paths()["include"], '-DLOCO_BUILT_FOR="%s"' % binding_for(), BINDING_DEPS[0], "-o", tmp, "-L" + HERE, "-lloco_layer_b200",
                           "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, BINDING)


def build(force: bool = False, verbose: bool = False) -> str:
    """Build what is out of date (everything with `force`); returns the path of libloco_b200.so."""
    wanted = []                                          # (library, its units)
    if force or stale():
        wanted.append((LIB, units()))
    if force or stale(LAYER_LIB, LAYER_DEPS):
        wanted.append((LAYER_LIB, [(s[:-3], s, []) for s in LAYER_SOURCES]))
    binding = force or stale_binding()
    if not wanted:
        if binding:
            build_binding()
        return LIB
    nvcc = nvcc_path()
    extra = ["-Xptxas", "-v"] if verbose else []
    with tempfile.TemporaryDirectory(prefix="loco_build_") as tmpdir:
        def compile_one(u):
            name, src, defs = u
            obj = os.path.join(tmpdir, name + ".o")
            subprocess.check_call([nvcc, *NVCC_FLAGS, *extra, *defs, "-c", os.path.join(CSRC, src), "-o", obj])
            return obj

        with ThreadPoolExecutor(max_workers=max(1, os.cpu_count() or 1)) as ex:
            jobs = [(lib, [ex.submit(compile_one, u) for u in us]) for lib, us in wanted]
            for lib, futures in jobs:
                objs = [f.result() for f in futures]
                tmp = lib + ".tmp.%d" % os.getpid()
                subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static",
                                       "-Xcompiler", "-fPIC", "-o", tmp, *objs])
                os.replace(tmp, lib)
    if binding:
        build_binding()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
