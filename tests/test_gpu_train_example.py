"""The example that runs the operators together: MXFP4 products forward and
backward, one clipping norm, the projected step and AdamW."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_mxfp4.py")


def test_training_lowers_the_loss():
    """A fifth of the first loss after 200 steps."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("train_mxfp4", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    first, last = mod.train(200)
    assert last < 0.2 * first, (first, last)
