"""The ctypes binding without torch: a process that brings its own pointers and streams."""
import os
import subprocess
import sys

from paper_2609_33614_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
sys.modules["torch"] = None  # an import of torch fails
from paper_2609_33614_gb300 import eat


class Buffer:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        return self.at


a = [Buffer(4096 * i) for i in range(1, 5)]
assert eat.lib().eat_balance_workspace(64, 8) > 0
try:
    eat.eat_rms_norm(a[0], None, 0, 64, eat.EAT_BF16, a[1], 1e-6, None, a[2], eat.EAT_BF16, stream=0)
except eat.EatError as e:
    assert e.status == eat.EAT_ERR_INVALID_ARG and "T >= 1" in str(e)
else:
    raise SystemExit("no error")
print("fine")
"""


def test_the_ctypes_binding_needs_no_torch():
    build.build()
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr
