"""A learner in few bits for the actors in few bits: `python examples/low_bit_learner.py` on a GPU.

Behaviour cloning: a student policy (67 observations, three hidden layers of 256 units with LayerNorm + tanh behind the first, 21
tanh actions) learns the actions of a fixed full-precision one on seeded observations.  Every product of its training step runs
on the library's learner's operators:

  forward   y = Q4(x) W4^T + b on microscaled 4-bit floats; LayerNorm; what the backward pass needs is kept in 8 bits
  backward  the weights' gradients from the 8-bit checkpoints, the inputs' through the 4-bit weights, LayerNorm's from its checkpoint
            (a ReLU's mask is that of its input, in full)

The weights themselves, their updates (Adam) and what is element by element (tanh, ReLU, the loss) are torch's, in fp32.  In the
end the student acts for one observation at a time on its 4-bit layers, and is handed to the 8-bit actor as any policy is.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1910_01055_amd import binding as aq  # noqa: E402
from paper_1910_01055_amd import synth  # noqa: E402

DEV = "cuda:0"


class Layer:
    """One fully connected layer in 4 bits with what follows it, its checkpoints and its gradients."""

    def __init__(self, p, act, eps, batch, dtype):
        self.w, self.b = (torch.from_numpy(p[k]).to(DEV) for k in ("w", "b"))
        n, k = self.w.shape
        self.act, self.eps, self.n, self.k = act, eps, n, k
        self.q = aq.mx4_empty(n, k)
        self.kept_in = aq.ckpt8_empty(batch, k)
        self.z = torch.empty(batch, n, dtype=dtype, device=DEV)
        self.dx = torch.empty(batch, k, dtype=dtype, device=DEV)
        self.dw, self.db = torch.empty_like(self.w), torch.empty_like(self.b)
        self.params, self.grads = [self.w, self.b], [self.dw, self.db]
        sizes = [aq.mx4_linear_workspace(batch, n, k), aq.ckpt8_weight_grad_workspace(batch, n, k), aq.mx4_input_grad_workspace(batch, n, k)]
        if act == "ln_tanh":
            self.gamma, self.beta = (torch.from_numpy(p[k]).to(DEV) for k in ("gamma", "beta"))
            self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
            self.params += [self.gamma, self.beta]
            self.grads += [self.dgamma, self.dbeta]
            self.normed, self.dz = torch.empty_like(self.z), torch.empty_like(self.z)
            self.mean, self.rstd = torch.empty(batch, device=DEV), torch.empty(batch, device=DEV)
            self.kept_z = aq.ckpt8_empty(batch, n)
            sizes.append(aq.layernorm_backward_workspace(batch, n))
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device=DEV) if max(sizes) else None

    def quantize(self):
        aq.mx4_quantize(self.w, self.q)

    def forward(self, x):
        aq.ckpt8_pack(x, self.kept_in)
        aq.mx4_linear(x, self.q, self.b, self.z, self.ws)
        if self.act == "relu":
            return torch.relu(self.z)
        if self.act == "ln_tanh":
            aq.layernorm_forward(self.z, self.gamma, self.beta, self.eps, self.normed, self.mean, self.rstd, self.kept_z)
            return torch.tanh(self.normed)
        return self.z

    def backward(self, dy, kept_out, first):
        """dy: the gradient of what forward returned, which the next layer keeps as `kept_out`."""
        if self.act == "relu":  # (of z itself: small positive values are zeros in a checkpoint)
            dy = dy * (self.z > 0)
        elif self.act == "ln_tanh":
            h = torch.empty_like(self.z)
            aq.ckpt8_unpack(kept_out, h)
            dn = dy * (1 - h * h)
            aq.layernorm_backward(dn, self.kept_z, self.gamma, self.mean, self.rstd, self.dz, self.dgamma, self.dbeta, self.ws)
            dy = self.dz
        aq.ckpt8_weight_grad(dy, self.kept_in, self.dw, self.db, self.ws)
        if first:
            return None
        aq.mx4_input_grad(dy, self.q, self.dx, self.ws)
        return self.dx

    def act_one(self, x):
        """Few rows, without anything kept."""
        y = torch.empty(x.shape[0], self.n, dtype=x.dtype, device=DEV)
        size = aq.mx4_linear_workspace(x.shape[0], self.n, self.k)
        aq.mx4_linear(x, self.q, self.b, y, torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)
        if self.act == "ln_tanh":
            z = y
            y = torch.empty_like(z)
            aq.layernorm_forward(z, self.gamma, self.beta, self.eps, y)
            return torch.tanh(y)
        return torch.relu(y) if self.act == "relu" else y


class Student:
    def __init__(self, net, batch, dtype=torch.bfloat16, seed=9000):
        self.net = net
        self.layers = [Layer(p, l["act"], net["ln_eps"], batch, dtype) for p, l in zip(synth.make_params(net, seed=seed), net["layers"])]
        self.params = [p for l in self.layers for p in l.params]
        self.adam = torch.optim.Adam(self.params, lr=1e-3)

    def step(self, obs, target):
        """One training step; the loss as a device scalar."""
        x = obs
        for l in self.layers:
            l.quantize()
            x = l.forward(x)
        a = torch.tanh(x.float())
        e = a - target
        dy = (2.0 / e.numel() * e * (1 - a * a)).to(x.dtype)
        for i in reversed(range(len(self.layers))):
            kept_out = self.layers[i + 1].kept_in if i + 1 < len(self.layers) else None
            dy = self.layers[i].backward(dy, kept_out, first=i == 0)
        for l in self.layers:
            for p, g in zip(l.params, l.grads):
                p.grad = g
        self.adam.step()
        return (e * e).mean()

    def act(self, obs):
        for l in self.layers:
            l.quantize()
        x = obs
        for l in self.layers:
            x = l.act_one(x)
        return torch.tanh(x.float())

    def arrays(self):
        """Weights, biases, gains and offsets as the policy's entry points take them."""
        ln = [l.act == "ln_tanh" for l in self.layers]
        return ([l.w for l in self.layers], [l.b for l in self.layers], [l.gamma if has else None for l, has in zip(self.layers, ln)],
                [l.beta if has else None for l, has in zip(self.layers, ln)])


def run(steps=300, batch=2048, tell=print):
    """(loss of the first steps, of the last ones, the 4-bit student's and its 8-bit actor's error on new observations)."""
    net = synth.net_config("cfg2")
    teacher = aq.Policy(net)
    teacher.policy_set_params_fp32(*aq.upload_params(synth.make_params(net, nonzero_bias=True)))
    student = Student(net, batch)
    losses = []
    for i in range(steps):
        obs = aq.to_dev(synth.make_obs(net, batch, seed=100_000 + i))
        target = torch.empty(batch, synth.action_dim(net), device=DEV)
        teacher.policy_forward_fp32(obs, target)
        losses.append(student.step(obs.to(torch.bfloat16), target))
        if i % 50 == 0 or i == steps - 1:
            tell(f"step {i}: loss {float(losses[-1]):.5f}")
    losses = torch.stack(losses).cpu()
    # new observations: one at a time on the 4-bit layers, all at once on the 8-bit actor
    obs = aq.to_dev(synth.make_obs(net, 256, seed=7))
    target = torch.empty(256, synth.action_dim(net), device=DEV)
    teacher.policy_forward_fp32(obs, target)
    one = torch.cat([student.act(obs[i:i + 1].to(torch.bfloat16)) for i in range(16)])
    error4 = float(((one - target[:16]) ** 2).mean())
    actor = aq.Policy(net)
    arrays = student.arrays()
    actor.policy_set_params_fp32(*arrays)
    actor.quantize_params(*arrays, actor.calibrate_fp32(obs))
    actions = torch.empty_like(target)
    actor.policy_forward_int8(obs, actions)
    error8 = float(((actions - target) ** 2).mean())
    tell(f"error on new observations: 4-bit student, one at a time {error4:.5f}; its 8-bit actor {error8:.5f}")
    teacher.close()
    actor.close()
    return float(losses[:10].mean()), float(losses[-10:].mean()), error4, error8


if __name__ == "__main__":
    run()
