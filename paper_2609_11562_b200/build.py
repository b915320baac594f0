"""Builds the C-ABI library in-tree with nvcc for sm_100a (libentwine.so next to this file), and with the C compiler the
extension module that marshals the operators' arguments (_opcalls.so)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libentwine.so")
OPCALLS = os.path.join(HERE, "_opcalls.so")
INCLUDE = os.path.join(ROOT, "include")
SOURCES = ["plan.cc", "entwine_kernels.cu", "quant.cu", "moe.cu", "gemm_i8.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


STAMP = LIB + ".srchash"


def _source_hash() -> str:
    """Hash of everything the library is built from (file times do not survive a copy of the tree)."""
    import hashlib
    h = hashlib.sha256()
    deps = sorted(os.path.join(d, f) for d in (CSRC, INCLUDE) for f in os.listdir(d))
    for d in deps:
        h.update(os.path.basename(d).encode())
        with open(d, "rb") as f:
            h.update(f.read())
    h.update(os.environ.get("ENTWINE_NVCC_FLAGS", "").encode())
    return h.hexdigest()


def needs_build() -> bool:
    if not all(os.path.exists(f) for f in (LIB, OPCALLS, STAMP)):
        return True
    with open(STAMP) as f:
        return f.read().strip() != _source_hash()


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC",
             "-I", INCLUDE, "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    flags += os.environ.get("ENTWINE_NVCC_FLAGS", "").split()
    with tempfile.TemporaryDirectory() as tmp:
        # the sources side by side, then one link
        objs = [os.path.join(tmp, src + ".o") for src in SOURCES]
        cmds = [[_nvcc(), *flags, "-x", "cu", "-c", os.path.join(CSRC, src), "-o", obj] for src, obj in zip(SOURCES, objs)]
        cmds.append([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I",
                     sysconfig.get_paths()["include"], os.path.join(CSRC, "opcalls.c"), "-o", OPCALLS])
        cmds = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in cmds]
        outs = [(p.communicate()[0], p.returncode) for p in cmds]
        if all(rc == 0 for _, rc in outs):
            res = subprocess.run([_nvcc(), *flags, "-shared", *objs, "-o", LIB], capture_output=True, text=True)
            outs.append((res.stdout + res.stderr, res.returncode))
    for text, rc in outs:
        if verbose or rc != 0:
            sys.stderr.write(text)
    if any(rc != 0 for _, rc in outs):
        raise RuntimeError("building libentwine.so or _opcalls.so failed")
    with open(STAMP, "w") as f:
        f.write(_source_hash() + "\n")
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
