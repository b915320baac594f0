"""CPU tests of the build: what it does where the operators' marshalling module cannot be built."""
import os
import shutil
import subprocess
import sys
import sysconfig

import pytest

from conftest import ROOT
from paper_2609_11562_b200 import build as B

B.build()


@pytest.fixture
def tree(tmp_path):
    """A copy of the package with its built library and without the marshalling module."""
    shutil.copytree(B.HERE, tmp_path / "paper_2609_11562_b200", ignore=shutil.ignore_patterns("__pycache__", "_opcalls*"))
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    return tmp_path


def _python(tree, code, **env):
    return subprocess.run([sys.executable, "-c", code], cwd=tree, env={**os.environ, **env}, capture_output=True, text=True, timeout=300)


USE = """
from paper_2609_11562_b200 import build as B
lib = open(B.LIB, 'rb').read()
assert B.build() == B.LIB and open(B.LIB, 'rb').read() == lib     # the library is not built again
from paper_2609_11562_b200 import entwine as E
assert E.Plan(1024, 512, 128, 4, E.ORDER_INTERLEAVED, 4).counts()['n_reduce'] > 0
try:
    E.quant_i8([[1.0]], None, None)
except (ImportError, E.EntwineError) as e:
    print(type(e).__name__, e)
"""


@pytest.mark.parametrize("compiler", ["false", "no-such-compiler"])
def test_the_library_stands_without_the_marshalling_module(tree, compiler):
    r = _python(tree, USE, CC=compiler)
    assert r.returncode == 0, r.stderr
    assert "building _opcalls failed" in r.stderr
    assert r.stdout.startswith("ImportError") and "could not be loaded" in r.stdout and "cannot import name" in r.stdout
    r = _python(tree, USE)                    # with a compiler that works it is built, and the operators answer
    assert r.returncode == 0 and r.stdout.startswith("EntwineError"), r.stderr


def test_a_module_of_other_sources_is_not_left_in_place(tree):
    assert _python(tree, USE).stdout.startswith("EntwineError")
    with open(tree / "paper_2609_11562_b200" / "csrc" / "opcalls.c", "a") as f:
        f.write("/* changed */\n")
    r = _python(tree, USE, CC="false")
    assert r.stdout.startswith("ImportError"), r.stderr


def test_the_module_is_named_for_its_interpreter(tree):
    """One that any interpreter would load is taken away, and the files are put in place whole."""
    package = tree / "paper_2609_11562_b200"
    (package / "_opcalls.so").write_bytes(b"built by another interpreter")
    assert _python(tree, USE).stdout.startswith("EntwineError")
    built = sorted(f.name for f in package.iterdir() if f.name.endswith(".so"))
    assert built == ["_opcalls" + sysconfig.get_config_var("EXT_SUFFIX"), "libentwine.so"]


def test_a_rebuilt_module_does_not_touch_the_loaded_one(tree):
    """The module's file is replaced, not written over: the loaded one keeps its own."""
    r = _python(tree, USE + """
import os
old = os.open(B.OPCALLS, os.O_RDONLY)
before = os.read(old, 1 << 24)
B._build_opcalls()
os.lseek(old, 0, 0)
assert os.read(old, 1 << 24) == before and os.fstat(old).st_ino != os.stat(B.OPCALLS).st_ino
""")
    assert r.returncode == 0, r.stderr
