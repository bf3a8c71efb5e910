"""The example that runs the operators behind the decode together: the student's loss falls."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_student_learns():
    spec = importlib.util.spec_from_file_location("distill_fidelity", os.path.join(ROOT, "examples", "distill_fidelity.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.run(steps=30, images=24, say=lambda line: None)
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.8 * losses[0], losses
