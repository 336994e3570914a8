"""The training example end to end: the operators together, as a user runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_loss_falls():
    spec = importlib.util.spec_from_file_location("train_draft", os.path.join(ROOT, "examples", "train_draft.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.main(steps=12, rows=200, d=256, f=512, V_full=5000, verbose=False)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
    assert m.main(steps=3, rows=200, d=256, f=512, V_full=5000, verbose=False) == losses[:3]      # the same run twice
