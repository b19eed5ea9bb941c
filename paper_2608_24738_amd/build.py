"""Builds ``libtm_edt.so`` (the HIP kernels and C-ABI) in place with hipcc for gfx950, and ``_torch_ops.so`` (torch
functions with gradients that call it) with the host compiler."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libtm_edt.so")
SOURCES = [os.path.join(PKG, "csrc", "edt_host.hip"),
           os.path.join(PKG, "csrc", "train", "train_host.hip"),
           os.path.join(PKG, "csrc", "train", "head_host.hip"),
           os.path.join(PKG, "csrc", "train", "rows_host.hip")]
TORCH_OPS = os.path.join(PKG, "_torch_ops.so")
TORCH_SOURCE = os.path.join(PKG, "csrc", "train", "torch_ops.cpp")
DEPS = SOURCES + [TORCH_SOURCE] + sorted(glob.glob(os.path.join(PKG, "csrc", "*.h"))) + sorted(
    glob.glob(os.path.join(PKG, "csrc", "train", "*.h"))) + [
    os.path.join(ROOT, "include", "tm_edt.h"), os.path.join(ROOT, "include", "tm_train.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # packed fp32 VALU forms are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _torch_flags():
    """What compiles and links a source against the installed torch: (compile, link)."""
    import torch
    root = os.path.dirname(torch.__file__)
    compile_flags = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
                     "-DTORCH_EXTENSION_NAME=_torch_ops",
                     "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    for path in (os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                 "/opt/rocm/include", sysconfig.get_paths()["include"]):
        compile_flags += ["-isystem", path]
    link_flags = ["-L", os.path.join(root, "lib"), "-lc10", "-lc10_hip", "-ltorch", "-ltorch_cpu", "-ltorch_python",
                  "-L", PKG, "-ltm_edt", "-Wl,-rpath,$ORIGIN"]
    return compile_flags, link_flags


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cxx = os.environ.get("CXX", "g++")
    tmp = LIB + ".tmp%d" % os.getpid()
    tmp_ops = TORCH_OPS + ".tmp%d" % os.getpid()
    # the sources share no device code: each is compiled by itself, all at once
    objects = [tmp + "%d.o" % i for i in range(len(SOURCES))]
    torch_object = tmp_ops + ".o"
    torch_compile, torch_link = _torch_flags()
    cmds = [[hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
            for src, obj in zip(SOURCES, objects)]
    cmds.append([cxx, *torch_compile, "-c", TORCH_SOURCE, "-o", torch_object])
    links = [([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objects], tmp, LIB),
             ([cxx, "-shared", "-o", tmp_ops, torch_object, *torch_link], tmp_ops, TORCH_OPS)]
    if verbose:
        print("\n".join(" ".join(cmd) for cmd in cmds + [link for link, _, _ in links]), flush=True)
    try:
        running = [subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for cmd in cmds]
        outputs = [proc.communicate()[0] for proc in running]
        if any(proc.returncode != 0 for proc in running):
            sys.stderr.write("".join(outputs))
            raise RuntimeError("compiling libtm_edt.so failed")
        for link, made, target in links:
            res = subprocess.run(link, capture_output=True, text=True)
            if res.returncode != 0:
                sys.stderr.write(res.stdout + res.stderr)
                raise RuntimeError("linking %s failed" % os.path.basename(target))
            os.replace(made, target)
    finally:
        for obj in objects + [torch_object]:
            if os.path.exists(obj):
                os.remove(obj)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(TORCH_OPS):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(TORCH_OPS))
    return any(os.path.getmtime(d) > t for d in DEPS)


if __name__ == "__main__":
    print(build(verbose=True))
