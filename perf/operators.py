"""The learner's operators, as cases with stated sizes: LayerNorm with its backward pass, 8-bit activation checkpoints with the
gradients that read them, and layers whose products run on microscaled 4-bit floats.

A learner trains the policy that the 8-bit actors run.  Its forward pass normalises, keeps what the backward pass needs in 8 bits
and multiplies in 4; its backward pass reads the checkpoints and the 4-bit weights again.  The same 4-bit layers serve single
observations.  Every case goes through the binding, one call at a time on torch's current stream, as a program that uses the
library does.

Formats (blocks are 32 values along a row; the last one of a row may be short):
  checkpoint   x ~ code * 2^(scale - 133), code in [-127, 127] to nearest even, scale - 127 = floor(log2(max |x| of the block))
  4-bit float  x ~ value * 2^(scale - 127), value in 0, .5, 1, 1.5, 2, 3, 4, 6 with a sign, to nearest even and at most 6,
               scale - 125 = floor(log2(max |x| of the block)); two to a byte, the even one in the low half
A scale is one byte, at least 0; a block that holds a NaN or an infinity has 255 and stands for NaNs.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # the normalised layer of one actor's policy on one observation: nothing but latency
        {"do": "ln_forward", "rows": 1, "cols": 256, "type": "f32", "name": "ln forward b1"},
        # one learner batch through the control policy's normalised layer, forward and backward
        {"do": "ln_train", "rows": 4096, "cols": 256, "type": "f32", "ckpt": False, "name": "ln train control b4096"},
        # the wide policy's layer over as many rows as a replay sweep feeds, the input kept in 8 bits
        {"do": "ln_train", "rows": 65536, "cols": 1024, "type": "bf16", "ckpt": True, "name": "ln train wide b65536"},
        # first layer of the control policy: observations kept in 8 bits, weight gradient in full precision
        {"do": "weight_grad", "rows": 4096, "k": 67, "n": 256, "type": "f32", "name": "weight grad control b4096"},
        # the widest layer of the paper's policies over a large batch
        {"do": "weight_grad", "rows": 65536, "k": 2048, "n": 2048, "type": "bf16", "name": "weight grad fc2048 b65536"},
        # 4-bit weights of one layer, from the learner's fp32 ones
        {"do": "quantize", "rows": 2048, "cols": 2048, "type": "f32", "name": "mx4 weights 4M"},
        # activations of odd sizes, in half precision
        {"do": "quantize", "rows": 3001, "cols": 777, "type": "f16", "name": "mx4 ragged 3001x777"},
        # one observation through a 2048-wide layer
        {"do": "linear", "rows": 1, "k": 2048, "n": 2048, "type": "bf16", "name": "mx4 linear fc2048 b1"},
        # some hundred environments through a layer of odd sizes
        {"do": "linear", "rows": 300, "k": 1111, "n": 403, "type": "f32", "name": "mx4 linear ragged b300"},
        # a product that fills the chip
        {"do": "linear", "rows": 16384, "k": 4096, "n": 4096, "type": "bf16", "name": "mx4 linear 4096 b16384"},
        # the gradient that goes on through a 2048-wide layer of 4-bit weights
        {"do": "input_grad", "rows": 8192, "k": 2048, "n": 2048, "type": "bf16", "name": "input grad fc2048 b8192"},
        # the same for a small batch behind the layer of odd sizes
        {"do": "input_grad", "rows": 300, "k": 1111, "n": 403, "type": "f16", "name": "input grad ragged b300"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Log-uniform; half of the larger ones are multiples of 32."""
    n = _log(rng, lo, hi)
    return n if n < 64 or rng.random() < 0.5 else n // 32 * 32


def draw(rng):
    do = rng.choice(["ln_forward", "ln_train", "ln_train", "weight_grad", "weight_grad", "quantize", "linear", "linear", "linear",
                     "input_grad"])
    kind = rng.choice(["f32", "f16", "bf16", "bf16"])
    if do in ("ln_forward", "ln_train", "quantize"):
        cols = _size(rng, 16, 8192)
        case = {"do": do, "rows": _size(rng, 1, min(65536, (1 << 25) // cols)), "cols": cols, "type": kind}
        return dict(case, ckpt=rng.random() < 0.5) if do == "ln_train" else case
    k, n = _size(rng, 16, 4096), _size(rng, 8, 4096)
    most = (1 << 37) // (2 if kind == "f32" else 1)
    return {"do": do, "rows": _size(rng, 1, max(1, min(65536, (1 << 26) // max(k, n), most // (k * n)))), "k": k, "n": n, "type": kind}


def work(case):
    e, do = BYTES[case["type"]], case["do"]
    if do in ("ln_forward", "ln_train", "quantize"):
        m, c = case["rows"], case["cols"]
        if do == "ln_forward":
            return {"bytes": 2 * m * c * e + 8 * c + 8 * m, "flops": 8 * m * c}
        if do == "ln_train":  # x, dy in; y, dx out; gains, offsets and their gradients; the rows' statistics
            return {"bytes": 4 * m * c * e + 16 * c + 8 * m, "flops": 24 * m * c}
        return {"bytes": m * c * (e + 4), "flops": 4 * m * c}
    m, k, n = case["rows"], case["k"], case["n"]
    w4 = n * (16 + 1) * ((k + 31) // 32)
    if do == "linear":
        return {"bytes": m * (k + n) * e + w4 + 4 * n, "flops": 2 * m * k * n}
    if do == "input_grad":
        return {"bytes": m * (k + n) * e + w4, "flops": 2 * m * k * n}
    return {"bytes": m * (k + n) * e + 4 * n * k + 4 * n, "flops": 2 * m * k * n + m * n}


# ---- the plain forms

def _blocks(x):
    """fp32 [rows][blocks][32] (zeros behind the last value) and floor(log2) of each block's largest magnitude, int32;
    a block that is not finite is told by the third."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    x = x.float()
    if nb * 32 != cols:
        x = torch.cat([x, x.new_zeros(rows, nb * 32 - cols)], 1)
    x = x.view(rows, nb, 32)
    amax = x.abs().amax(2)
    bad = ~(amax < math.inf)
    top = (torch.where(bad, torch.ones_like(amax), amax).view(torch.int32) >> 23) - 127
    return x, top, bad


def _pow2(e):
    """2^e in fp32 for -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _scaled(x, e):
    """x * 2^-e, e in [-133, 127] for each block, in two exact steps."""
    half = e >> 1
    return x * _pow2(-half)[:, :, None] * _pow2(half - e)[:, :, None]


def plain_ckpt8(x):
    """What the 8-bit checkpoint of x stands for, fp32."""
    b, top, bad = _blocks(x)
    e = top.clamp(min=-127) - 6
    v = torch.round(_scaled(b, e)).clamp(-127, 127)
    v = torch.where(bad[:, :, None], torch.full_like(v, math.nan), _scaled(v, -e))
    return v.view(x.shape[0], -1)[:, :x.shape[1]]


def plain_mx4(x):
    """4-bit codes of x, two to a byte, and the blocks' scales."""
    b, top, bad = _blocks(x)
    scale = (top + 125).clamp(min=0)
    s = _scaled(b, scale - 127)
    a = s.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    code = (code + 8 * (s < 0).int()).to(torch.uint8)
    code = torch.where(bad[:, :, None], torch.zeros_like(code), code).view(x.shape[0], -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), torch.where(bad, torch.full_like(scale, 255), scale).to(torch.uint8)


def plain_mx4_values(codes, scales, cols):
    """What 4-bit codes stand for, fp32."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1, 32)
    v = _scaled(table[c.int()], 127 - scales.int())
    v = torch.where((scales == 255)[:, :, None], torch.full_like(v, math.nan), v)
    return v.view(codes.shape[0], -1)[:, :cols]


def plain_layernorm(x, gamma, beta):
    x = x.float()
    mean = x.sum(1) / x.shape[1]
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / x.shape[1] + EPS)
    return d * rstd[:, None] * gamma + beta, mean, rstd


def plain_layernorm_backward(dy, x, gamma, mean, rstd):
    dy = dy.float()
    h = (x.float() - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    n = x.shape[1]
    dx = rstd[:, None] * (g - g.sum(1, keepdim=True) / n - h * ((g * h).sum(1, keepdim=True) / n))
    return dx, (dy * h).sum(0), dy.sum(0)


# ---- inputs

def _inputs(case, seed):
    """The inputs of a case: a dict of tensors, from the seed alone."""
    g = torch.Generator(device=DEV).manual_seed(1_000_003 * (seed + 1))
    t = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    do = case["do"]
    if do in ("ln_forward", "ln_train"):
        m, c = case["rows"], case["cols"]
        # rows of their own spread and offset, as pre-activations have
        s = {"x": (normal(m, c) * torch.exp(0.5 * normal(m, 1)) + 0.5 * normal(m, 1)).to(t),
             "gamma": 1.0 + 0.1 * normal(c), "beta": 0.1 * normal(c)}
        if do == "ln_train":
            s["dy"] = (0.1 * normal(m, c)).to(t)
        return s
    if do == "quantize":
        m, c = case["rows"], case["cols"]
        return {"x": (normal(m, c) * torch.exp(0.5 * normal(m, 1)) / math.sqrt(c)).to(t)}
    m, k, n = case["rows"], case["k"], case["n"]
    if do == "weight_grad":
        # what leaves a ReLU, each unit with a spread of its own; a tenth of the units are silent
        unit = torch.exp(0.5 * normal(k)) * (torch.rand(k, generator=g, device=DEV) > 0.1)
        return {"x": (torch.relu(normal(m, k)) * unit).to(t), "dy": (0.1 * normal(m, n)).to(t)}
    w = normal(n, k) / math.sqrt(k)
    codes, scales = plain_mx4(w)
    if do == "linear":
        return {"x": normal(m, k).to(t), "codes": codes, "scales": scales, "bias": 0.1 * normal(n)}
    return {"dy": (0.1 * normal(m, n)).to(t), "codes": codes, "scales": scales}


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if not own:
        return s
    from paper_1910_01055_amd import binding as aq
    do, t = case["do"], TYPES[case["type"]]
    f32 = torch.float32

    def new(*shape, dtype=t):
        return torch.empty(shape, dtype=dtype, device=DEV)

    def workspace(n):
        return new(n, dtype=torch.uint8)

    s["aq"] = aq
    if do in ("ln_forward", "ln_train"):
        m, c = case["rows"], case["cols"]
        s.update(y=new(m, c), mean=new(m, dtype=f32), rstd=new(m, dtype=f32), kept=None)
        if do == "ln_train":
            s.update(dx=new(m, c), dgamma=new(c, dtype=f32), dbeta=new(c, dtype=f32), kept=aq.ckpt8_empty(m, c) if case["ckpt"] else None,
                     ws=workspace(aq.layernorm_backward_workspace(m, c)))
    elif do == "quantize":
        m, c = case["rows"], case["cols"]
        s.update(q=aq.mx4_empty(m, c), values=new(m, c, dtype=f32))
    else:
        m, k, n = case["rows"], case["k"], case["n"]
        if do == "weight_grad":
            s.update(kept=aq.ckpt8_empty(m, k), dw=new(n, k, dtype=f32), db=new(n, dtype=f32), ws=workspace(aq.ckpt8_weight_grad_workspace(m, n, k)))
        else:
            s["w"] = aq.Mx4(s["codes"], s["scales"], k)
            if do == "linear":
                s.update(y=new(m, n), ws=workspace(aq.mx4_linear_workspace(m, n, k)))
            else:
                s.update(dx=new(m, k), ws=workspace(aq.mx4_input_grad_workspace(m, n, k)))
    return s


def run(s):
    return (_run_own if own else _run_plain)(s, s["case"]["do"])


def _run_own(s, do):
    aq = s["aq"]
    if do == "ln_forward":
        aq.layernorm_forward(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if do == "ln_train":
        aq.layernorm_forward(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"], s["kept"])
        aq.layernorm_backward(s["dy"], s["kept"] or s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return s["y"], s["dx"], s["dgamma"], s["dbeta"]
    if do == "weight_grad":
        aq.ckpt8_pack(s["x"], s["kept"])
        aq.ckpt8_weight_grad(s["dy"], s["kept"], s["dw"], s["db"], s["ws"])
        return s["dw"], s["db"]
    if do == "quantize":
        aq.mx4_quantize(s["x"], s["q"])
        aq.mx4_dequantize(s["q"], s["values"])
        return s["values"]
    if do == "linear":
        aq.mx4_linear(s["x"], s["w"], s["bias"], s["y"], s["ws"])
        return s["y"]
    aq.mx4_input_grad(s["dy"], s["w"], s["dx"], s["ws"])
    return s["dx"]


def _run_plain(s, do):
    t = TYPES[s["case"]["type"]]
    if do == "ln_forward":
        y, mean, rstd = plain_layernorm(s["x"], s["gamma"], s["beta"])
        return y.to(t), mean, rstd
    if do == "ln_train":
        y, mean, rstd = plain_layernorm(s["x"], s["gamma"], s["beta"])
        kept = plain_ckpt8(s["x"]) if s["case"]["ckpt"] else s["x"]
        dx, dgamma, dbeta = plain_layernorm_backward(s["dy"], kept, s["gamma"], mean, rstd)
        return y.to(t), dx.to(t), dgamma, dbeta
    if do == "weight_grad":
        dy = s["dy"].float()
        return dy.t() @ plain_ckpt8(s["x"]), dy.sum(0)
    if do == "quantize":
        codes, scales = plain_mx4(s["x"])
        return plain_mx4_values(codes, scales, s["case"]["cols"])
    w = plain_mx4_values(s["codes"], s["scales"], s["case"]["k"])
    if do == "linear":
        codes, scales = plain_mx4(s["x"])
        return (plain_mx4_values(codes, scales, s["case"]["k"]) @ w.t() + s["bias"]).to(t)
    return (s["dy"].float() @ w).to(t)


# ---- the definitions in 64 bits

def _exact_blocks(x, levels):
    """x rounded by blocks of 32: `levels(a)` rounds magnitudes below 2 in units of the power of two at or below the largest."""
    rows, cols = x.shape
    out = torch.zeros(rows, (cols + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    out[:, :cols] = x.double()
    out = out.view(rows, -1, 32)
    most = out.abs().amax(2, keepdim=True)
    unit = torch.exp2(torch.frexp(most)[1].double() - 1.0)  # most = m 2^e with m in [1/2, 1)
    out = torch.where(most > 0, torch.sign(out) * levels(out.abs() / unit) * unit, torch.zeros_like(out))
    return out.view(rows, -1)[:, :cols]


def _ckpt_levels(a):
    return torch.clamp(torch.round(a * 64.0), max=127.0) / 64.0


def _mx4_levels(a):
    a = 4.0 * a  # the largest in [4, 8)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.clamp(torch.round(a / step) * step, max=6.0) / 4.0


def exact(case, seed):
    s, do = _inputs(case, seed), case["do"]
    d = {k: v.double() for k, v in s.items() if v.is_floating_point()}
    if do in ("ln_forward", "ln_train"):
        x = d["x"]
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        rstd = (var + EPS).rsqrt()
        y = (x - mean) * rstd * d["gamma"] + d["beta"]
        if do == "ln_forward":
            return y, mean[:, 0], rstd[:, 0]
        h = ((_exact_blocks(x, _ckpt_levels) if case["ckpt"] else x) - mean) * rstd
        g = d["dy"] * d["gamma"]
        dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * rstd
        return y, dx, (d["dy"] * h).sum(0), d["dy"].sum(0)
    if do == "weight_grad":
        return torch.matmul(d["dy"].t().contiguous(), _exact_blocks(d["x"], _ckpt_levels)), d["dy"].sum(0)
    if do == "quantize":
        return _exact_blocks(d["x"], _mx4_levels)
    value = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0, 8.0, 12.0], dtype=torch.float64, device=DEV) / 2.0
    c = torch.empty(case["n"], 2 * s["codes"].shape[1], dtype=torch.int64, device=DEV)
    c[:, 0::2], c[:, 1::2] = s["codes"] % 16, s["codes"] // 16
    w = value[c % 8] * (1 - 2 * (c // 8))
    w = (w * torch.exp2(s["scales"].double() - 127.0).repeat_interleave(32, 1))[:, :case["k"]]
    if do == "linear":
        return torch.matmul(_exact_blocks(d["x"], _mx4_levels), w.t().contiguous()) + d["bias"]
    return torch.matmul(d["dy"], w)
