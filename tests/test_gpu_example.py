"""The example of the handle-free operators with the optimizer: a 4-bit student learns from a stored teacher."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_student_learns():
    path = os.path.join(ROOT, "examples", "distill_4bit_student.py")
    spec = importlib.util.spec_from_file_location("distill_4bit_student", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, generated = example.train(steps=40, workers=2, vocab=301, hidden=128, layers=1, tokens=256, top=16)
    assert len(losses) == 40 and all(x == x and x < float("inf") for x in losses)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5]), (losses[:5], losses[-5:])
    assert len(generated) == 8 and all(0 <= t < 301 for t in generated)
