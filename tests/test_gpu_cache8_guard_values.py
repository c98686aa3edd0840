"""Guard bands around the decode over the 8-bit cache, and its results' values, with both builds (see cache8_guard_values_run.py)."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("debug", ["0", "1"])
def test_results_between_guard_bands(debug):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_17644_b200 import build
    build.build(debug=(debug == "1"))
    out = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "cache8_guard_values_run.py")], env=dict(os.environ, LAGA_DEBUG=debug),
                         capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout[-1500:] + out.stderr[-3000:]
    assert "GUARD_VALUES_OK" in out.stdout
