"""The learner's operators together, as a program uses them: the example trains a policy on them and hands it to the 8-bit actor."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_low_bit_learner(aq):
    spec = importlib.util.spec_from_file_location("low_bit_learner", os.path.join(ROOT, "examples", "low_bit_learner.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, error4, error8 = example.run(steps=120, batch=1024, tell=lambda s: print(s, flush=True))
    # it learns: the loss falls to a third; and what acts is what was trained
    assert last < first / 3
    assert error4 < first / 2 and error8 < first / 2
