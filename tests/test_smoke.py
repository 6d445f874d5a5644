"""The smoke run, in a process of its own: it needs no solver library of torch's, which may not be there."""
import ast
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


def test_smoke_calls_no_decomposition():
    tree = ast.parse((ROOT / "__graft_entry__.py").read_text())
    assert not [n.attr for n in ast.walk(tree) if isinstance(n, ast.Attribute) and n.attr in ("linalg", "svd", "qr")]


@pytest.mark.gpu
def test_smoke():
    code = "import __graft_entry__ as g; g.smoke(); assert 'cuda_linalg' not in open('/proc/self/maps').read()"
    run = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "smoke ok" in run.stdout, run.stdout + run.stderr
