"""The example that runs norm, layers, head, perplexity signal and balance loss together."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_lm_loop_learns(capsys):
    from paper_2609_33614_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location(
        "lm_loop", os.path.join(ROOT, "examples", "lm_loop.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    history = m.main(["--steps", "8"])
    assert all(math.isfinite(v) for v in history)
    # 64 distinct contexts with fixed successors: the head finds them within a few steps
    assert history[-1] < 0.7 * history[0]
    assert "perplexity" in capsys.readouterr().out
