"""examples/ffn_q8.py: the operators together, as a program uses them."""
import importlib.util
import os

import pytest

from gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_ffn_q8_example():
    require_gpu()
    spec = importlib.util.spec_from_file_location("ffn_q8", os.path.join(ROOT, "examples", "ffn_q8.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    got = m.main("vig_ti", 60)
    # rounding to 8 bits: a step is top / 127 and top three or four deviations, so each
    # rounded factor is off by about 1 / (127 sqrt 12) * 3.5 = 0.8 %, four in a row
    assert 0.002 < got["ffn"] < 0.04
    # the norm's part of the difference goes, the rounding's stays
    assert got["sizes"][0] > 0.1 and got["sizes"][-1] < 0.03
