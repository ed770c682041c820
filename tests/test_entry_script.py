"""The build and smoke entry points as a script."""
import ast
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ENTRY = os.path.join(ROOT, "__graft_entry__.py")


def test_the_script_runs_when_all_is_defined():
    with open(ENTRY) as f:
        body = ast.parse(f.read()).body
    guards = [i for i, n in enumerate(body) if isinstance(n, ast.If) and "__name__" in ast.dump(n.test)]
    assert guards == [len(body) - 1]


@pytest.mark.gpu
def test_smoke_as_a_script():
    r = subprocess.run([sys.executable, ENTRY, "smoke"], capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0 and "smoke ok" in r.stdout, r.stdout[-500:] + r.stderr[-2000:]
