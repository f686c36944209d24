"""GPU: the example's scoring after further training steps."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_scores_follow_the_training():
    """A window scored after a step is scored by the vocabulary matrix of that step, whether or not
    there was a score before it."""
    from paper_2609_33614_gb300 import build, eat
    build.build()
    spec = importlib.util.spec_from_file_location(
        "lm_loop_state", os.path.join(ROOT, "examples", "lm_loop.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    model = m.Model()
    tokens, targets, mask = m.batch(0)
    model.score(tokens, targets)
    for step in range(3):
        model.train_step(*m.batch(step))
        seen = {}
        q8, scale8 = m.e4m3_rows(model.head_w)
        head = eat.EatHead(q8, m.BATCH, w_scale=scale8)
        norm = eat.rms_norm_fp8

        def record(*a, **k):
            seen["rows"] = norm(*a, **k)
            return seen["rows"]

        eat.rms_norm_fp8 = record
        try:
            nll = model.score(tokens, targets)
        finally:
            eat.rms_norm_fp8 = norm
        q, scale, _ = seen["rows"]
        assert torch.equal(nll, head.nll(q, targets, x_scale=scale)[0])
        head.close()
    model.close()
