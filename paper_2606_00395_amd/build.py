"""Builds libpr2.so (HIP for gfx950) in-tree with hipcc.

Each translation unit compiles to an object under ``_build/`` in parallel,
then one shared library is linked next to this file, and beside it the binding's
compiled argument checks (``_args``, against the installed torch).  Always recompiles.
The library needs hipcc alone; where the checks do not compile (no g++, no headers of
the interpreter or of torch), none are left and the binding takes its own in Python.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpr2.so")
ARGS = os.path.join(HERE, "_args.so")
SOURCES = ["api.hip", "router.hip", "permute.hip", "gemm.hip", "tile.hip", "backward.hip",
           "predictor.hip", "noalloc.hip", "policy.hip", "dispatch.hip", "pack.hip", "wgrad.hip"]

HIPCC = os.environ.get("HIPCC", shutil.which("hipcc") or "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def _run(cmd):
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in p.stdout.splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    return p.returncode, out


def _args_command(out: str):
    """The binding's argument checks: host code on the interpreter's and torch's C++ API."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-isystem", sysconfig.get_paths()["include"],
            "-isystem", os.path.join(root, "include"), os.path.join(CSRC, "args.cpp"),
            "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", out]


def build_args() -> bool:
    """Builds ``_args``, or takes an older one away and says why there is none."""
    tmp = ARGS + ".tmp"
    try:
        cmd = _args_command(tmp)
        rc, out = _run(cmd)
    except (OSError, ImportError, AttributeError) as e:
        rc, out = 1, str(e)
    if rc == 0:
        os.replace(tmp, ARGS)
        return True
    for path in (tmp, ARGS):
        if os.path.exists(path):
            os.remove(path)
    print(out, file=sys.stderr)
    print("compiled argument checks not built; the binding's Python ones are used", file=sys.stderr)
    return False


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    objs = []
    cmds = []
    for src in SOURCES:
        obj = os.path.join(BUILD, src.replace(".hip", ".o"))
        objs.append(obj)
        cmds.append([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    with ThreadPoolExecutor(len(cmds) + 1) as ex:
        args = ex.submit(build_args)
        results = list(ex.map(_run, cmds))
        args.result()
    for cmd, (rc, out) in zip(cmds, results):
        if verbose or rc != 0:
            if out.strip():
                print(out, file=sys.stderr)
        if rc != 0:
            raise RuntimeError("hipcc failed: " + " ".join(cmd))
    tmp = LIB + ".tmp"
    rc, out = _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
    if rc != 0:
        print(out, file=sys.stderr)
        raise RuntimeError("link failed")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
