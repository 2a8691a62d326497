"""The package imports where torch does not: building and the C side need
none."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("error", ["ImportError('no torch')", "OSError('libtorch.so: cannot open shared object file')"])
def test_without_a_torch_that_loads(tmp_path, error):
    (tmp_path / "torch.py").write_text(f"raise {error}\n")
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([str(tmp_path), ROOT]))
    code = "import paper_2606_24031_amd as w4; from paper_2606_24031_amd import build; " \
           "print(w4.torch, w4.strerror(w4.ESHAPE))"
    r = subprocess.run([sys.executable, "-c", code], env=env, cwd=tmp_path, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.startswith("None "), r.stderr
