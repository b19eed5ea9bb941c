"""Builds ``libtm_edt.so`` (the HIP kernels and C-ABI) in place with hipcc for gfx950, and ``_torch_ops.so`` (torch
functions with gradients that call it) with the host compiler."""
from __future__ import annotations

import glob
import importlib.util
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


def _run(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(running, what: str) -> None:
    outputs = [proc.communicate()[0] for proc in running]
    if any(proc.returncode != 0 for proc in running):
        sys.stderr.write("".join(outputs))
        raise RuntimeError(what + " failed")


def build(verbose: bool = False) -> str:
    """Builds both. The library needs hipcc alone: it is there also where the torch functions cannot be built, which raises."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cxx = os.environ.get("CXX", "g++")
    tmp = LIB + ".tmp%d" % os.getpid()
    tmp_ops = TORCH_OPS + ".tmp%d" % os.getpid()
    # the sources share no device code: each is compiled by itself, all at once
    objects = [tmp + "%d.o" % i for i in range(len(SOURCES))]
    torch_object = tmp_ops + ".o"

    def start(cmds):
        if verbose:
            print("\n".join(" ".join(cmd) for cmd in cmds), flush=True)
        return [_run(cmd) for cmd in cmds]

    running, torch_running, missing = [], [], None
    try:
        running = start([[hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
                         for src, obj in zip(SOURCES, objects)])
        try:
            torch_compile, torch_link = _torch_flags()
            torch_running = start([[cxx, *torch_compile, "-c", TORCH_SOURCE, "-o", torch_object]])
        except (ImportError, OSError) as err:
            missing = err
        _finish(running, "compiling libtm_edt.so")
        _finish(start([[hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objects]]), "linking libtm_edt.so")
        os.replace(tmp, LIB)
        if missing is not None:
            raise RuntimeError("_torch_ops.so needs torch and a host compiler: %s" % missing) from missing
        _finish(torch_running, "compiling _torch_ops.so")
        _finish(start([[cxx, "-shared", "-o", tmp_ops, torch_object, *torch_link]]), "linking _torch_ops.so")
        os.replace(tmp_ops, TORCH_OPS)
    finally:
        for proc in running + torch_running:
            if proc.returncode is None:
                proc.communicate()
        for path in objects + [torch_object, tmp, tmp_ops]:
            if os.path.exists(path):
                os.remove(path)
    return LIB


def _torch_changed() -> float:
    """When the installed torch last changed, 0 without one."""
    spec = importlib.util.find_spec("torch")
    version = os.path.join(os.path.dirname(spec.origin), "version.py") if spec and spec.origin else ""
    return os.path.getmtime(version) if os.path.exists(version) else 0.0


def is_stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(TORCH_OPS):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(TORCH_OPS))
    return any(os.path.getmtime(d) > t for d in DEPS) or _torch_changed() > os.path.getmtime(TORCH_OPS)


if __name__ == "__main__":
    print(build(verbose=True))
