"""Gated layers, the recurrence and the optimizer together, as a program uses them: the example of a policy with a memory."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("recurrent_learner", os.path.join(ROOT, "examples", "recurrent_learner.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype,bits", [(torch.bfloat16, 8), (torch.float16, 8), (torch.float32, 32)])
def test_it_runs(aq, example, dtype, bits):
    policy, losses = example.run(steps=12, count=20, most=50, dtype=dtype, bits=bits, tell=lambda s: None)
    assert bool(torch.isfinite(losses).all()) and policy.steps == 12
    for name, w in policy.w.items():
        assert bool(torch.isfinite(w.float()).all()), name
        assert torch.equal(w, policy.master[name].to(w.dtype)), name  # the copies that the forward pass reads are the weights


def test_its_gradients(aq, example):
    """In fp32, against automatic differentiation of the same policy in 64 bits, step by step."""
    policy = example.RecurrentPolicy(dtype=torch.float32, bits=32, seed=3)
    count = 9
    x, offsets, starts, _ = example.replayed(count, 30, 16, 4, seed=5)
    g = torch.Generator().manual_seed(9)
    first, da = torch.randn(count, policy.units, generator=g), torch.randn(x.shape[0], 4, generator=g)
    policy.forward(x.to("cuda:0"), offsets.to("cuda:0"), starts.to("cuda:0"), first.to("cuda:0"))
    dfirst = policy.backward(da.to("cuda:0"))
    w = {k: v.cpu().double().requires_grad_() for k, v in policy.master.items()}
    state0 = first.double().requires_grad_()
    a = x.double() @ w["wg"].t()
    h = a * torch.sigmoid(a) * (x.double() @ w["wu"].t())
    f, v = torch.sigmoid(h @ w["wz"].t() + w["bz"]), h @ w["wv"].t()
    ys = []
    for s in range(count):
        y = state0[s]
        for t in range(int(offsets[s]), int(offsets[s + 1])):
            y = f[t] * (y * 0.0 if starts[t] else y) + (1 - f[t]) * v[t]
            ys.append(y)
    (torch.stack(ys) @ w["wo"].t() * da.double()).sum().backward()
    # fp32 values behind some hundred roundings each, sums of some hundred of them: 100 * 2^-24 of their size, in the 2-norm
    for name, got in list(policy.grad.items()) + [("first", dfirst)]:
        want = state0.grad if name == "first" else w[name].grad
        off = float((got.cpu().double() - want).norm() / want.norm())
        assert off < 100 * 2.0 ** -24, (name, off)


def test_it_acts_as_it_learned(aq, example):
    """One step at a time gives the actions that the whole sequence gives: the same values but for the roundings of the type, of which the
    products' inputs and outputs have one each."""
    policy, _ = example.run(steps=2, count=8, most=40, tell=lambda s: None)
    x, offsets, starts, _ = example.replayed(1, 150, 16, 4, seed=77)
    x, starts = x.to("cuda:0").to(policy.dtype), starts.to("cuda:0")
    whole = policy.forward(x, offsets.to("cuda:0"), starts, torch.zeros(1, policy.units, device="cuda:0"))
    one = example.act_one_by_one(policy, x, starts)
    assert float((one.float() - whole.float()).norm() / whole.float().norm()) < 4 * 2.0 ** -8
