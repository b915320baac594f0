"""CPU tests of what importing the binding needs."""
import subprocess
import sys

from conftest import ROOT
from paper_2609_11562_b200 import build as B

B.build()


def _python(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)


NO_TORCH = """
import importlib.abc, sys
class Refuse(importlib.abc.MetaPathFinder):
    def find_spec(self, name, path, target=None):
        if name.split('.')[0] == 'torch':
            raise ImportError('no torch here')
sys.meta_path.insert(0, Refuse())
"""


def test_plans_with_raw_addresses_need_no_torch():
    r = _python(NO_TORCH + """
from paper_2609_11562_b200 import entwine as E
p = E.Plan(1024, 512, 128, 4, E.ORDER_INTERLEAVED, 4)
assert p.counts()['n_reduce'] > 0
assert p.heap_bytes()[0] > 0 and E._ptr(1 << 20) == 1 << 20 and E._stream(7) == 7
assert 'torch' not in sys.modules
try:
    E.quant_i8(None, None, None, stream=0)      # the operators take torch tensors
except ImportError as e:
    assert 'no torch here' in str(e)
else:
    raise SystemExit('an operator ran without torch')
print('ok')
""")
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr


def test_importing_the_binding_does_not_import_torch():
    r = _python("import sys\nfrom paper_2609_11562_b200 import entwine\nprint('torch' in sys.modules)")
    assert r.stdout.strip() == "False", r.stderr


def test_operators_follow_a_reloaded_binding():
    """After a reload the operators raise the new module's error, although they were bound to the old one's."""
    r = _python("""
import importlib
from paper_2609_11562_b200 import entwine as E
for _ in range(2):
    try:
        E.quant_i8([[1.0]], None, None, stream=0)
    except E.EntwineError as e:
        assert e.code == E.ERR_INVALID
    E = importlib.reload(E)
print('ok')
""")
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr
