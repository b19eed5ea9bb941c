"""Builds ``libtm_edt.so`` (the HIP kernels and C-ABI) in place with hipcc for gfx950."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libtm_edt.so")
SOURCES = [os.path.join(PKG, "csrc", "edt_host.hip"),
           os.path.join(PKG, "csrc", "train", "train_host.hip")]
DEPS = SOURCES + sorted(glob.glob(os.path.join(PKG, "csrc", "*.h"))) + sorted(
    glob.glob(os.path.join(PKG, "csrc", "train", "*.h"))) + [
    os.path.join(ROOT, "include", "tm_edt.h"), os.path.join(ROOT, "include", "tm_train.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # packed fp32 VALU forms are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    # the sources share no device code: each is compiled by itself, all at once
    objects = [tmp + "%d.o" % i for i in range(len(SOURCES))]
    cmds = [[hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
            for src, obj in zip(SOURCES, objects)]
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objects]
    if verbose:
        print("\n".join(" ".join(cmd) for cmd in cmds + [link]), flush=True)
    try:
        running = [subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for cmd in cmds]
        outputs = [proc.communicate()[0] for proc in running]
        if any(proc.returncode != 0 for proc in running):
            sys.stderr.write("".join(outputs))
            raise RuntimeError("hipcc failed building libtm_edt.so")
        res = subprocess.run(link, capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError("hipcc failed linking libtm_edt.so")
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    os.replace(tmp, LIB)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in DEPS)


if __name__ == "__main__":
    print(build(verbose=True))
