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


def test_units_whose_checkpoint_rounds_to_nothing_learn(aq):
    """A ReLU's derivative is one for every positive value, also for those that the checkpoint of what it returns holds as zero."""
    import torch

    spec = importlib.util.spec_from_file_location("low_bit_learner", os.path.join(ROOT, "examples", "low_bit_learner.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    batch, n, k = 3, 32, 40
    w = torch.zeros(n, k)
    w[0, 0], w[1:30, 0], w[30, 0] = 1.0, 2.0 ** -10, -1.0  # outputs 1, 2^-10, -1 and 0
    layer = example.Layer({"w": w.numpy(), "b": torch.zeros(n).numpy()}, "relu", 0.0, batch, torch.float32)
    x = torch.zeros(batch, k, device="cuda:0")
    x[:, 0] = 1.0
    layer.quantize()
    kept_out = aq.ckpt8_empty(batch, n)
    aq.ckpt8_pack(layer.forward(x), kept_out)
    assert not bool(kept_out.codes[:, 1:].any())  # as the test is meant
    dx = layer.backward(torch.ones(batch, n, device="cuda:0"), kept_out, first=False)
    live = torch.zeros(n, device="cuda:0")
    live[:30] = batch
    assert torch.equal(layer.dw[:, 0], live) and not bool(layer.dw[:, 1:].any()) and torch.equal(layer.db, live)
    assert torch.equal(dx[:, 0], torch.full((batch,), 1.0 + 29 * 2.0 ** -10, device="cuda:0")) and not bool(dx[:, 1:].any())
