"""AdamW over all tensors of a policy against its definition in 64 bits.

Tolerances, U the rounding of an fp32 operation: the gradient's scale is off by three roundings (the norm, a division, its product), each
moment by its constants, products and sum: 8 U of the sum of its terms' magnitudes; the root of v by half of v's and one; a step by
those and seven roundings more (the root's correction, a product, eps, the division, the rate, its product, the weight's sum)."""
import math

import pytest
import torch

from paper_1910_01055_amd import binding as B
from test_gpu_learner import DEV, OUT, TYPES, U

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, WD = 3e-3, 0.9, 0.999, 1e-8, 0.02
PLACE, TURN = 0xC13FA9A9, 0x9E3779B9


class Tensor:
    """One tensor with its state, every part `at` elements into a buffer that is watched behind and in front."""

    def __init__(self, n, g_kind="f32", bits=32, copy=None, decay=True, at=0, seed=0, spread=2.0):
        g = torch.Generator().manual_seed(1000 * seed + n)
        self.n, self.bits, self.kind, self.copy_kind, self.decay = n, bits, g_kind, copy, decay
        scale = torch.exp(spread * torch.randn(n, generator=g))
        self.frames = []
        self.w = self.put(torch.randn(n, generator=g), at)
        self.g = self.put((1e-2 * torch.randn(n, generator=g) * scale).to(TYPES[g_kind]), at)
        self.copy = None if copy is None else self.put(torch.zeros(n, dtype=TYPES[copy]), at)
        m, v = 3e-3 * torch.randn(n, generator=g) * scale, 1e-4 * scale * scale * torch.rand(n, generator=g)
        if bits == 32:
            self.m, self.v = self.put(m, at), self.put(v, at)
        else:
            self.m, self.v = B.moment8_zeros(n, DEV), B.moment8_zeros(n, DEV)
            wide = B.Learned(self.w, self.g, m.to(DEV), v.to(DEV)) if n else None
            if n:
                B.moments_convert(B.LearnedSet([wide]), B.LearnedSet([B.Learned(self.w, self.g, self.m, self.v)]))
        self.learned = B.Learned(self.w, self.g, self.m, self.v, self.copy, decay)

    def put(self, values, at):
        buf = torch.full((at + values.numel() + 40,), 77.0, dtype=values.dtype, device=DEV)
        buf[at:at + values.numel()] = values.to(DEV)
        self.frames.append((buf, at, at + values.numel()))
        return buf[at:at + values.numel()]

    def moments(self):
        """m and v that are kept, in 64 bits on the host."""
        if self.bits == 32:
            return self.m.cpu().double(), self.v.cpu().double()
        return moment_values(self.m, self.n, 3), moment_values(self.v, self.n, 4) ** 2

    def unhurt(self):
        for buf, a, b in self.frames:
            assert bool((buf[:a] == 77.0).all()) and bool((buf[b:] == 77.0).all()), "values around a tensor were written"


def moment_values(q, n, bits):
    """What codes stand for: sqrt(v) for the second moment."""
    c = q.codes.cpu().long().view(-1, 32)
    sign = torch.where(c >> 7 > 0, -1.0, 1.0) if bits == 3 else torch.ones(c.shape)
    c = c & 127 if bits == 3 else c
    e, f = (c >> bits).double(), (c % (1 << bits)).double()
    x = torch.where(e > 0, (f + (1 << bits)) * torch.exp2(e - 15 - bits), f * 2.0 ** (-14 - bits))
    s = q.scales.cpu().double()[:, None]
    return torch.where(s == 255, torch.full_like(x, math.nan), sign.double() * x * torch.exp2(s - 127)).view(-1)[:n]


def check_moment8(q, n, want, tol, bits, step, half, what, nearest=False):
    """Codes of magnitudes `want`, known up to tol, as the definition has them."""
    blocks = (n + 31) // 32
    x = torch.zeros(32 * blocks, dtype=torch.float64)
    t = torch.zeros(32 * blocks, dtype=torch.float64)
    x[:n], t[:n] = want.abs(), tol
    x, t = x.view(-1, 32), t.view(-1, 32)
    scales = q.scales.cpu().double()[:, None]
    most, slack = x.amax(1, keepdim=True), t.amax(1, keepdim=True)
    unit = torch.exp2(scales - 127)
    assert bool(((most + slack >= unit) | (scales == 0)).all()) and bool((most - slack < 2 * unit).all()), f"{what}: scales"
    place = torch.arange(32 * blocks)
    turn = (place * PLACE + step * TURN + half * (1 << 31)) % (1 << 32)
    cut = 23 - bits
    d = torch.full(x.shape, 0.5, dtype=torch.float64) if nearest else (torch.div(turn, 1 << (32 - cut), rounding_mode="floor").double() / 2.0 ** cut).view(-1, 32)
    c = q.codes.cpu().long().view(-1, 32)
    if bits == 3:
        signs = torch.zeros(32 * blocks, dtype=torch.bool)
        signs[:n] = want < 0
        sure = (x > t) & (c & 127 > 0)
        assert bool(((c >> 7 > 0) == signs.view(-1, 32))[sure].all()), f"{what}: signs"
        c = c & 127

    def code(v):
        v = v.clamp(min=0.0) / unit
        e = torch.clamp(torch.floor(torch.log2(v.clamp(min=1e-300))), min=-14.0)
        e = torch.where(v < torch.exp2(e), e - 1, torch.where(v >= torch.exp2(e + 1), e + 1, e)).clamp(min=-14.0)
        step_of = torch.exp2(e - bits)
        up = torch.floor(v / step_of + d)  # in steps of this binade; one that is full is the next one's first
        return torch.clamp(up + (e + 14) * (1 << bits), max=float((16 << bits) - 1)), v

    lo, _ = code(x * (1 - 2 * U) - t)
    hi, v = code(x * (1 + 2 * U) + t)
    if bits == 4:
        lo, hi = (torch.where((x > 0) & (k == 0), torch.ones_like(k), k) for k in (lo, hi))
    ok = (c >= lo) & (c <= hi)
    assert bool(ok.all()), f"{what}: {int((~ok).sum())} of {ok.numel()} codes"
    assert bool((c.view(-1)[n:] == 0).all()), f"{what}: padding"
    assert float((lo != hi).double().mean()) < 0.02, f"{what}: nothing was checked"


def expected(t, scale, step, lr=LR):
    """(w, m, v), their tolerances and the copy's type, from the tensor's present state."""
    g = t.g.cpu().double() * scale
    m0, v0 = t.moments()
    w0 = t.w.cpu().double()
    m, v = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g
    mt = 8 * U * (B1 * m0.abs() + (1 - B1) * g.abs()) + 2.0 ** -140
    vt = 12 * U * v + 2.0 ** -140
    c1, c2 = 1 - B1 ** step, 1 - B2 ** step
    den = torch.sqrt(v / c2) + EPS
    up = lr / c1 * m / den
    decay = 1 - lr * WD if t.decay else 1.0
    w = w0 * decay - up
    wt = lr / c1 * mt / den + 20 * U * up.abs() + 3 * U * w0.abs()
    return (w, wt), (m, mt), (v, vt)


def close(got, want, what):
    off = (got - want[0]).abs()
    assert bool((off <= want[1]).all()), f"{what}: {float((off - want[1]).max())} over"


def check(tensors, step, scale=1.0, max_norm=math.inf, norm=None, **how):
    want = [expected(t, scale, how.get("number", step), how.get("rate", LR)) for t in tensors]
    B.adamw_step(B.LearnedSet([t.learned for t in tensors]), how.get("lr", LR), B1, B2, EPS, WD, how.get("d_step", step), norm, max_norm)
    torch.cuda.synchronize()
    for i, (t, (w, m, v)) in enumerate(zip(tensors, want)):
        close(t.w.cpu().double(), w, f"w {i}")
        if t.bits == 32:
            close(t.m.cpu().double(), m, f"m {i}")
            close(t.v.cpu().double(), v, f"v {i}")
        elif t.n:
            check_moment8(t.m, t.n, m[0], m[1], 3, how.get("number", step), 0, f"m {i}")
            r = torch.sqrt(v[0])
            check_moment8(t.v, t.n, r, 8 * U * r + 2.0 ** -70, 4, how.get("number", step), 1, f"v {i}")
        if t.copy is not None:
            assert bool((t.copy == t.w.to(t.copy.dtype)).all()), f"copy {i}"
        t.unhurt()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind,copy", [("f32", None), ("f16", "bf16"), ("bf16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("n", [1, 7, 8, 31, 32, 33, 250, 2047, 2048, 2049, 10000])
def test_one_tensor(bits, kind, copy, n):
    t = Tensor(n, kind, bits, copy, at=3 if n % 2 else 0, seed=bits)
    for step in (1, 2, 1000):
        check([t], step)


@pytest.mark.parametrize("count", [1, 39, 40, 41, 130])
def test_many_tensors(count):
    """More than one launch's worth, of mixed kinds, some of them without values."""
    kinds = ["f32", "f16", "bf16"]
    tensors = [Tensor((i * 37) % 300 if i % 7 else 0, kinds[i % 3], 8 if i % 2 else 32, [None, "bf16", "f16"][i % 3], i % 5 != 0, i % 4, seed=i)
               for i in range(count)]
    check(tensors, 3)
    check(tensors, 4)


@pytest.mark.parametrize("bits", [32, 8])
def test_norm_and_clipping(bits):
    tensors = [Tensor(n, k, bits, seed=9) for n, k in ((5000, "f32"), (33, "f16"), (0, "f32"), (70001, "bf16"))]
    tensors = [t for t in tensors if t.n or bits == 32]
    s = B.LearnedSet([t.learned for t in tensors])
    norm = torch.empty(1, device=DEV)
    size = B.grad_norm_workspace(s)
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    B.grad_norm(s, norm, ws)
    want = math.sqrt(sum(float((t.g.cpu().double() ** 2).sum()) for t in tensors))
    assert abs(float(norm) - want) <= 2 * U * want
    check(tensors, 5, scale=0.25, max_norm=0.25 * float(norm), norm=norm)
    check(tensors, 6, scale=1.0, max_norm=2.0 * float(norm), norm=norm)


def test_norm_of_many_values_and_of_none():
    """As many workgroups as there may be, values whose squares leave fp32, no values at all."""
    n = 2048 * 2100 + 5
    for value in (1.0, 1e25):
        t = B.Learned(torch.zeros(n, device=DEV), torch.full((n,), value, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV))
        s = B.LearnedSet([t])
        norm = torch.empty(1, device=DEV)
        B.grad_norm(s, norm, torch.empty(B.grad_norm_workspace(s), dtype=torch.uint8, device=DEV))
        exact = float(torch.tensor(value)) * math.sqrt(n)
        assert abs(float(norm) - exact) <= 2 * U * exact
    none = B.LearnedSet([])
    assert B.grad_norm_workspace(none) == 0
    B.grad_norm(none, norm)
    assert float(norm) == 0.0
    B.adamw_step(none, LR, B1, B2, EPS, WD, 1, norm, 1.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("norm", [math.inf, math.nan, -math.inf])
def test_a_norm_that_is_not_finite_leaves_everything(bits, norm):
    t = Tensor(100, "f32", bits, "bf16", seed=4)
    parts = [t.w, t.copy] + ([t.m, t.v] if bits == 32 else [t.m.codes, t.v.codes, t.m.scales, t.v.scales])
    before = [p.clone() for p in parts]
    B.adamw_step(B.LearnedSet([t.learned]), LR, B1, B2, EPS, WD, 1, torch.full((1,), norm, device=DEV), 1.0)
    assert all(bool((a == b).all()) for a, b in zip(before, parts))


def test_step_and_rate_on_the_device_in_a_graph():
    """A captured step whose number and rate change from replay to replay, two graphs of tensors of their own side by side."""
    tensors = [[Tensor(3000, "bf16", 8, "bf16", seed=1), Tensor(77, "f32", 32, seed=2)] for _ in range(2)]
    sets = [B.LearnedSet([t.learned for t in ts]) for ts in tensors]
    number, rate = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, device=DEV)
    norms = [torch.empty(1, device=DEV) for _ in sets]
    spaces = [torch.empty(B.grad_norm_workspace(s), dtype=torch.uint8, device=DEV) for s in sets]
    graphs = []
    for s, norm, ws in zip(sets, norms, spaces):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.grad_norm(s, norm, ws)
            B.adamw_step(s, rate, B1, B2, EPS, WD, number, norm, 1e30)
        graphs.append(graph)
    for step in (1, 2, 3, 100_000):
        number.fill_(step)
        rate.fill_(LR / step ** 0.25)
        lr = float(rate)
        want = [[expected(t, 1.0, step, lr) for t in ts] for ts in tensors]
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for ts, ws in zip(tensors, want):
            for t, (w, m, v) in zip(ts, ws):
                close(t.w.cpu().double(), w, f"w in step {step}")
                if t.bits == 32:
                    close(t.m.cpu().double(), m, f"m in step {step}")
                else:
                    check_moment8(t.m, t.n, m[0], m[1], 3, step, 0, f"m in step {step}")


@pytest.mark.parametrize("n", [1, 32, 1000, 5003])
def test_convert(n):
    """To 8 bits to the nearest code, and what it stands for back, both exactly."""
    t = Tensor(n, seed=3)
    m8, v8 = B.moment8_zeros(n, DEV), B.moment8_zeros(n, DEV)
    eight, wide = B.LearnedSet([B.Learned(t.w, t.g, m8, v8)]), B.LearnedSet([t.learned])
    m, v = t.moments()
    B.moments_convert(wide, eight)
    check_moment8(m8, n, m, torch.zeros(n, dtype=torch.float64), 3, 0, 0, "m", nearest=True)
    r = torch.sqrt(v)
    check_moment8(v8, n, r, 2 * U * r, 4, 0, 1, "v", nearest=True)
    B.moments_convert(eight, wide)
    assert bool((t.m.cpu().double() == moment_values(m8, n, 3)).all())
    assert bool((t.v.cpu().double() == (moment_values(v8, n, 4) ** 2).float().double()).all())
    codes = m8.codes.clone(), v8.codes.clone()
    B.moments_convert(wide, eight)  # values that codes stand for are kept
    assert bool((codes[0] == m8.codes).all()) and bool((codes[1] == v8.codes).all())
    t.unhurt()


def test_codes_are_right_on_the_mean():
    """What a code loses in one step it makes up for in others: over 256 steps from the same state, the mean of what is kept is what was
    to be kept, within a 50th of a step of the code (a sequence of multiples of an irrational number covers [0, 1) to log(256) / 256)."""
    n = 96
    g = torch.Generator().manual_seed(8)
    m0 = torch.randn(n, generator=g)
    grad = torch.zeros(n, device=DEV)
    w = torch.zeros(n, device=DEV)
    total = torch.zeros(n, dtype=torch.float64)
    m8, v8 = B.moment8_zeros(n, DEV), B.moment8_zeros(n, DEV)
    B.moments_convert(B.LearnedSet([B.Learned(w, grad, m0.to(DEV), torch.zeros(n, device=DEV))]), B.LearnedSet([B.Learned(w, grad, m8, v8)]))
    start = m8.codes.clone(), m8.scales.clone()
    kept = moment_values(m8, n, 3) * float(torch.tensor(B1, dtype=torch.float32))
    s = B.LearnedSet([B.Learned(w, grad, m8, v8)])
    for step in range(1, 257):
        m8.codes.copy_(start[0])
        m8.scales.copy_(start[1])
        B.adamw_step(s, 0.0, B1, B2, EPS, 0.0, step)
        total += moment_values(m8, n, 3)
    most = kept.abs().view(-1, 32).amax(1, keepdim=True)
    top = torch.exp2(torch.floor(torch.log2(most)))
    unit = torch.exp2(torch.floor(torch.log2(kept.abs().view(-1, 32))).maximum(torch.log2(top) - 14) - 3)
    off = (total / 256 - kept).abs().view(-1, 32) / unit
    assert float(off.max()) < 0.02, float(off.max())


def test_a_moment_that_is_not_finite():
    """A gradient's NaN reaches what it belongs to in 32 bits, and its block in 8."""
    for bits in (32, 8):
        t = Tensor(64, "f32", bits, seed=6)
        t.g[40] = math.nan
        check_w = t.w.clone()
        B.adamw_step(B.LearnedSet([t.learned]), LR, B1, B2, EPS, WD, 1)
        bad = torch.isnan(t.w)
        assert bool(bad[40]) and int(bad.sum()) == 1 and not bool((t.w[:32] == check_w[:32]).all())
        m, v = t.moments()
        want = torch.zeros(64, dtype=torch.bool)
        want[40 if bits == 32 else slice(32, 64)] = True
        assert bool((torch.isnan(m) == want).all()) and bool((torch.isnan(v) == want).all())
        B.adamw_step(B.LearnedSet([t.learned]), LR, B1, B2, EPS, WD, 2)
        assert bool((torch.isnan(t.w.cpu()) == want).all())


def test_on_another_stream():
    t = Tensor(5000, "bf16", 8, "bf16", seed=7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check([t], 2)
