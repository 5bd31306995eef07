"""The example that trains a gated block with AdamW on streamed buffers, as a program runs it."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_classifier.py")


def _example():
    spec = importlib.util.spec_from_file_location("gated_classifier", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [32, 8])
def test_a_gated_block_learns_what_softmax_regression_cannot(bits):
    """Labels of a gated block, ragged buffers and mini-batches.  The loss falls with every iteration and ends below that of the linear predictor."""
    losses, linear = _example().train(rows=20_011, p=64, hidden=256, buffers=3, batch=500, passes=2, iterations=4, state_bits=bits, say=lambda s: None)
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < linear


def test_runs_are_reproducible():
    m = _example()
    runs = [m.train(rows=3_000, p=40, hidden=72, classes=7, buffers=2, batch=333, passes=1, iterations=1, state_bits=8, say=lambda s: None) for _ in range(2)]
    assert runs[0] == runs[1]
