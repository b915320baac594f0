"""Builds the C-ABI library in-tree with nvcc for sm_100a (libentwine.so next to this file), and with the C compiler the
extension module that marshals the operators' arguments (_opcalls, for the running interpreter).

The library needs nothing of Python.  Where the module cannot be built (no Python.h), the library stands all the same, with
a warning: plans work, and the operators say why they do not."""
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
# named for this interpreter, whose binary interface it uses: another one finds none instead of a wrong one
OPCALLS = os.path.join(HERE, "_opcalls" + sysconfig.get_config_var("EXT_SUFFIX"))
UNTAGGED = os.path.join(HERE, "_opcalls.so")  # as it was once named: any interpreter would load it
OPCALLS_SOURCE = os.path.join(CSRC, "opcalls.c")
INCLUDE = os.path.join(ROOT, "include")
SOURCES = ["plan.cc", "entwine_kernels.cu", "quant.cu", "moe.cu", "gemm_i8.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


STAMP = LIB + ".srchash"
OPCALLS_STAMP = OPCALLS + ".srchash"


def _hash(files, *settings) -> str:
    """Hash of what a file is built from (file times do not survive a copy of the tree)."""
    import hashlib
    h = hashlib.sha256()
    for d in files:
        h.update(os.path.basename(d).encode())
        with open(d, "rb") as f:
            h.update(f.read())
    for v in settings:
        h.update(v.encode())
    return h.hexdigest()


def _source_hash() -> str:
    deps = sorted(os.path.join(d, f) for d in (CSRC, INCLUDE) for f in os.listdir(d))
    return _hash([d for d in deps if d != OPCALLS_SOURCE], os.environ.get("ENTWINE_NVCC_FLAGS", ""))


def _opcalls_hash() -> str:
    return _hash([OPCALLS_SOURCE])


def _stamped(built: str, stamp: str, want: str) -> bool:
    if not (os.path.exists(built) and os.path.exists(stamp)):
        return False
    with open(stamp) as f:
        return f.read().strip() == want


def _stamp(stamp: str, value: str) -> None:
    with open(stamp, "w") as f:
        f.write(value + "\n")


def _beside(path: str) -> str:
    """A name in the same folder, to build at before it takes the place of `path` at once: who loads that meanwhile has
    the old file or the new one, whole."""
    return os.path.join(HERE, f"tmp{os.getpid()}_{os.path.basename(path)}")


def needs_build() -> bool:
    return os.path.exists(UNTAGGED) or not (_stamped(LIB, STAMP, _source_hash()) and
                                            _stamped(OPCALLS, OPCALLS_STAMP, _opcalls_hash()))


def _build_library(verbose: bool) -> None:
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC",
             "-I", INCLUDE, "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    flags += os.environ.get("ENTWINE_NVCC_FLAGS", "").split()
    with tempfile.TemporaryDirectory() as tmp:
        # the sources side by side, then one link
        objs = [os.path.join(tmp, src + ".o") for src in SOURCES]
        cmds = [[_nvcc(), *flags, "-x", "cu", "-c", os.path.join(CSRC, src), "-o", obj] for src, obj in zip(SOURCES, objs)]
        cmds = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in cmds]
        outs = [(p.communicate()[0], p.returncode) for p in cmds]
        if all(rc == 0 for _, rc in outs):
            res = subprocess.run([_nvcc(), *flags, "-shared", *objs, "-o", _beside(LIB)], capture_output=True, text=True)
            outs.append((res.stdout + res.stderr, res.returncode))
    for text, rc in outs:
        if verbose or rc != 0:
            sys.stderr.write(text)
    if any(rc != 0 for _, rc in outs):
        raise RuntimeError("building libentwine.so failed")
    os.replace(_beside(LIB), LIB)
    _stamp(STAMP, _source_hash())


def _build_opcalls() -> None:
    """Leaves no module where it cannot build one: a stale one is not loaded in its place."""
    try:
        res = subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I",
                              sysconfig.get_paths()["include"], OPCALLS_SOURCE, "-o", _beside(OPCALLS)], capture_output=True, text=True)
        text, failed = res.stdout + res.stderr, res.returncode != 0
    except OSError as e:
        text, failed = f"{e}\n", True
    sys.stderr.write(text)
    for old in (UNTAGGED, UNTAGGED + ".srchash", *((OPCALLS_STAMP, OPCALLS) if failed else ())):
        if os.path.exists(old):
            os.remove(old)
    if failed:
        sys.stderr.write("warning: building _opcalls failed (above); libentwine.so stands, the operators of entwine_ops.h "
                         "cannot be called from Python\n")
        return
    os.replace(_beside(OPCALLS), OPCALLS)
    _stamp(OPCALLS_STAMP, _opcalls_hash())


def build(force: bool = False, verbose: bool = False) -> str:
    if force or not _stamped(LIB, STAMP, _source_hash()):
        _build_library(verbose)
    if force or os.path.exists(UNTAGGED) or not _stamped(OPCALLS, OPCALLS_STAMP, _opcalls_hash()):
        _build_opcalls()
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
