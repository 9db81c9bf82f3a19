"""Compiles the HIP library for gfx950 in-tree (paper_1509_05186_amd/lib/libetf.so)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIBDIR, "libetf.so")

SOURCES = ["etf_host.cpp", "etf_device.hip", "etf_build.hip", "etf_kv.hip", "etf_prompt.hip", "etf_pages.hip"]
HEADERS = ["etf_internal.h", "etf_launch.h", "etf_kernels.hip.h", "etf_ctx_kernels.hip.h", "etf_ivf.hip.h", "etf_prune_kernels.hip.h", "etf_build_kernels.hip.h", "etf_kv_types.hip.h", "etf_kv_kernels.hip.h", "etf_prompt_kernels.hip.h", "etf_pages_kernels.hip.h"]

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=gfx950",
    # packed-FP32 instructions are kept out of every kernel (generated by the compiler from plain
    # float code otherwise)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-pthread",
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(ROOT, "include", "etf.h")]
    return any(os.path.getmtime(p) > t for p in deps)


def build_library(force: bool = True, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    os.makedirs(LIBDIR, exist_ok=True)
    tmp = LIB + ".tmp%d" % os.getpid()
    common = [hipcc()] + [f for f in FLAGS if f != "-shared"] + os.environ.get("ETF_EXTRA_FLAGS", "").split()
    common += ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    # one compiler process per source, side by side; then one link
    objs, procs = [], []
    for src in SOURCES:
        obj = "%s.%s.o" % (tmp, os.path.splitext(src)[0])
        cmd = common + ["-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        objs.append(obj)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, pr in procs:
        out, _ = pr.communicate()
        if pr.returncode != 0:
            sys.stderr.write(out)
            failed = True
        elif verbose and out:
            print(out)
    try:
        if failed:
            raise RuntimeError("hipcc failed")
        link = [hipcc(), "-shared", "-fPIC", "--offload-arch=gfx950", "-pthread"] + objs + ["-o", tmp]
        if verbose:
            print(" ".join(link), flush=True)
        res = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout)
            raise RuntimeError("hipcc (link) failed")
    finally:
        for o in objs:
            if os.path.exists(o):
                os.remove(o)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
