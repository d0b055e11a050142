"""Build the CUDA library libecasq.so in-tree for sm_103a (nvcc, no cmake).

Each translation unit under csrc/ is compiled in parallel, then linked into
paper_2608_18147_gb300/_build/libecasq.so with the CUDA runtime linked
statically.  csrc/binding.c becomes a Python extension beside it (the C
compiler and Python's headers), which the operators on 4-bit codes alone need:
build_binding() makes it, at their first call if not before.
"""
from __future__ import annotations

import glob
import os
import shlex
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "_build")
LIB = os.path.join(OUT, "libecasq.so")
BINDING_SRC = os.path.join(CSRC, "binding.c")
BINDING = os.path.join(OUT, "_codes" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "--expt-relaxed-constexpr",
              "-Xcompiler", "-fPIC,-ffp-contract=off,-fno-fast-math", "-Xptxas", "-warn-spills"]


def nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    return "nvcc"


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + [os.path.join(HERE, "..", "include", "ecasq.h")]
    return any(os.path.getmtime(p) > t for p in deps if os.path.exists(p))


def build_binding(force: bool = False) -> str:
    """The Python extension of csrc/binding.c; its path."""
    deps = [p for p in (BINDING_SRC, os.path.join(HERE, "..", "include", "ecasq.h")) if os.path.exists(p)]
    if not force and os.path.exists(BINDING) and all(os.path.getmtime(BINDING) >= os.path.getmtime(p) for p in deps):
        return BINDING
    os.makedirs(OUT, exist_ok=True)
    tmp = BINDING + ".%d.tmp" % os.getpid()
    cmd = shlex.split(os.environ.get("CC") or "gcc") + ["-std=c11", "-O2", "-shared", "-fPIC", "-I" + sysconfig.get_paths()["include"],
                                                        BINDING_SRC, "-o", tmp]
    try:
        done = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    except OSError as e:
        raise RuntimeError("%s: %s" % (cmd[0], e)) from e
    if done.returncode != 0:
        raise RuntimeError("%s failed:\n%s" % (cmd[0], done.stdout.decode(errors="replace")))
    os.replace(tmp, BINDING)
    return BINDING


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    if not force and not _stale():
        return LIB
    os.makedirs(OUT, exist_ok=True)
    objs, procs = [], []
    for src in sources():
        obj = os.path.join(OUT, os.path.splitext(os.path.basename(src))[0] + ".o")
        cmd = [nvcc()] + ARCH + NVCC_FLAGS + list(extra_flags) + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    failed = []
    for src, pr in procs:
        out, _ = pr.communicate()
        text = out.decode(errors="replace")
        if pr.returncode != 0:
            failed.append((src, text))
        elif verbose and text.strip():
            print(text, file=sys.stderr)
    if failed:
        msg = "\n".join("%s:\n%s" % f for f in failed)
        raise RuntimeError("nvcc failed:\n" + msg)
    tmp = LIB + ".%d.tmp" % os.getpid()
    subprocess.run([nvcc()] + ARCH + ["-shared", "-cudart", "static", "-o", tmp] + objs, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
    print(build_binding(force="--force" in sys.argv))
