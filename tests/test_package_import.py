"""What an import of the package brings in."""

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def python(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)


def test_star_import_does_without_torch():
    """The simulator's modules come without torch; moe, which works on its
    tensors, is imported by name."""
    r = python("import sys; from paper_2505_01616_amd import *; netsim, program; assert 'torch' not in sys.modules")
    assert r.returncode == 0, r.stderr


def test_operators_by_name():
    r = python("from paper_2505_01616_amd import moe; moe.route, moe.Router")
    assert r.returncode == 0, r.stderr
