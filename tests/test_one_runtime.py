"""The library and torch share one HIP runtime, whichever a program uses first."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys
import paper_1909_05073_amd as P
for first in sys.argv[1:]:
    P.lib() if first == "library" else __import__("torch")
runtimes = {line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line}
assert len(runtimes) == 1, runtimes
"""


@pytest.mark.parametrize("order", [("library", "torch"), ("torch", "library")])
def test_one_runtime_is_loaded(order):
    r = subprocess.run([sys.executable, "-c", PROGRAM, *order], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
