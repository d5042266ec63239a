"""What the binding of the operators on floating-point activations must not ask of programs that do not use them."""
from __future__ import annotations

import os
import subprocess
import sys

from paper_2011_10680_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_handle_needs_no_torch():
    """Without torch a handle is made as before, or refused by the library for want of a GPU."""
    build.build()
    program = """
import sys
sys.modules["torch"] = None                    # importing it raises ImportError
from paper_2011_10680_b200 import binding
try:
    binding.Handle(0).close()
except binding.HqError:
    pass
print("no import")
"""
    done = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert done.returncode == 0 and "no import" in done.stdout, done.stderr[-2000:]
