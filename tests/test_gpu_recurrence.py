"""The gated linear recurrence against its definition in 64 bits, step by step.

Tolerances: U is the rounding of an fp32 operation.  A gate f = 1 / (1 + e^-|z|) (or e^-|z| times it) is off by at most E = (1.5 |z| + 6) U:
the exponent's product with log2(e) by |z| U 1.45 in all, the exponential and the reciprocal by two roundings each, an addition and a product
by one.  A state is a sum of products of gates with one term (1 - f) v, each term with a gate, a product and an addition for every step
that it lies back, in whatever order the steps are joined: with the sum a_t = f a_{t-1} + (1 - f) |v| of their magnitudes, its error is at most
b_t = f b_{t-1} + (E + 4 U) a_t.  What is rounded to a type has half a step of that type more."""
import pytest
import torch

import gated_shapes as shapes
from paper_1910_01055_amd import binding as B
from test_gpu_learner import DEV, OUT, SENTINEL, TINY, TYPES, U, Framed

pytestmark = pytest.mark.gpu


def oracle(z, v, first, offsets, starts):
    """h, the last states and their error bounds, the gates with theirs; all fp64 on the host."""
    rows, c = z.shape
    f, rest = torch.sigmoid(z), torch.sigmoid(-z)
    e = (1.5 * z.abs() + 6) * U
    h, hb = torch.zeros_like(v), torch.zeros_like(v)
    last, lastb = first.clone(), torch.zeros_like(first)
    for s in range(len(offsets) - 1):
        state, a, b = first[s], first[s].abs(), torch.zeros(c, dtype=torch.float64)
        for t in range(offsets[s], offsets[s + 1]):
            if starts is not None and starts[t]:
                state, a, b = state * 0, a * 0, b * 0
                state[:] = 0.0  # (whatever it was)
                a[:] = 0.0
                b[:] = 0.0
            state = f[t] * state + rest[t] * v[t]
            a = f[t] * a + rest[t] * v[t].abs()
            b = f[t] * b + (e[t] + 4 * U) * a
            h[t], hb[t] = state, b
        last[s], lastb[s] = state, b
    return h, hb, last, lastb, f, rest, e


def oracle_backward(dy, dlast, v, y, first, offsets, starts, f, rest, e):
    rows, c = v.shape
    out = {k: torch.zeros_like(v) for k in ("dz", "dv", "dzb", "dvb")}
    dfirst, dfirstb = dlast.clone(), torch.zeros_like(dlast)
    for s in range(len(offsets) - 1):
        G, a, b = dlast[s].clone(), dlast[s].abs(), torch.zeros(c, dtype=torch.float64)
        for t in reversed(range(offsets[s], offsets[s + 1])):
            cut = starts is not None and bool(starts[t])
            before = torch.zeros_like(G) if cut else y[t - 1] if t > offsets[s] else first[s]
            g, ga, gb = dy[t] + G, dy[t].abs() + a, b + U * (dy[t].abs() + a)
            slope = rest[t] * f[t] * (before - v[t])
            out["dv"][t], out["dvb"][t] = g * rest[t], rest[t] * (gb + (e[t] + 2 * U) * ga)
            out["dz"][t], out["dzb"][t] = g * slope, slope.abs() * (gb + (2 * e[t] + 6 * U) * ga)
            G, a, b = f[t] * g, f[t] * ga, f[t] * (gb + (e[t] + 3 * U) * ga)
            if cut:
                G, a, b = torch.zeros_like(G), torch.zeros_like(a), torch.zeros_like(b)
        dfirst[s], dfirstb[s] = G, b
    return out, dfirst, dfirstb


def near(got, want, bound, kind, what):
    tol = bound + OUT[kind] * (want.abs() + bound) + TINY[kind]
    off = (got - want).abs()
    assert bool((off <= tol).all()), f"{what}: {float((off - tol).max())} over at {int((off > tol).sum())} of {off.numel()}"


def run(offsets, rows, c, kind, starts_share=0.05, gap=0, at=0, seed=0, with_first=True, uniform=False, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    t = TYPES[kind]
    n = len(offsets) - 1
    z, v, dy = ((torch.randn(rows, c, generator=g) * k + o).to(t) for k, o in ((spread, 1.0), (1.0, 0.0), (0.1, 0.0)))
    first, dlast = (torch.randn(n, c, generator=g) * k for k in (0.5, 0.1))
    if not with_first:
        first, dlast = torch.zeros(n, c), torch.zeros(n, c)
    starts = (torch.rand(rows, generator=g) < starts_share).to(torch.uint8) if starts_share else None
    Z, V, DY = (Framed(rows, c, t, gap, at, x.to(DEV)) for x in (z, v, dy))
    Y, DZ, DV = (Framed(rows, c, t, gap, at) for _ in range(3))
    f32 = {"dtype": torch.float32, "device": DEV}
    last, dfirst = torch.full((n, c), SENTINEL, **f32), torch.full((n, c), SENTINEL, **f32)
    size = B.recurrence_workspace(rows, n, c)
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV) if size else None
    off = None if uniform else torch.tensor(offsets, dtype=torch.int32, device=DEV)
    st = None if starts is None else starts.to(DEV)
    d_first, d_dlast = (first.to(DEV), dlast.to(DEV)) if with_first else (None, None)
    B.recurrence_forward(Z.m, V.m, d_first, Y.m, last, off, st, ws)
    y = Y.get()
    used = torch.zeros(rows, dtype=torch.bool)
    used[offsets[0]:offsets[-1]] = True
    h, hb, want_last, lastb, f, rest, e = oracle(z.double(), v.double(), first.double(), offsets, starts)
    near(y[used], h[used], hb[used], kind, "y")
    assert bool((y[~used] == SENTINEL).all()), "rows outside of all sequences were written"
    near(last.cpu().double(), want_last, lastb, "f32", "last")
    B.recurrence_backward(DY.m, d_dlast, Z.m, V.m, Y.m, d_first, DZ.m, DV.m, dfirst, off, st, ws)
    out, want, wantb = oracle_backward(dy.double(), dlast.double(), v.double(), y, first.double(), offsets, starts, f, rest, e)
    for name, M in (("dz", DZ), ("dv", DV)):
        got = M.get()
        near(got[used], out[name][used], out[name + "b"][used], kind, name)
        assert bool((got[~used] == SENTINEL).all()), "gradients outside of all sequences were written"
    near(dfirst.cpu().double(), want, wantb, "f32", "dfirst")


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("c", [1, 2, 7, 64, 129, 256])
def test_ragged(kind, c):
    """Lengths from none to many tiles, two empty ones in a row, rows in front of the first and behind the last sequence."""
    lengths = [0, 1, 17, 2, 0, 0, 130, 33, 16, 64]
    offsets = [3]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    run(offsets, offsets[-1] + 5, c, kind, seed=c)


def lengths_of(count, mean, ragged):
    """As many rows in all; ragged ones from none to some times the mean, in no order."""
    if not ragged:
        return [mean] * count
    g = torch.Generator().manual_seed(count + mean)
    cuts = torch.randint(0, count * mean + 1, (count - 1,), generator=g).sort()[0].tolist()
    ends = [0] + cuts + [count * mean]
    return [b - a for a, b in zip(ends, ends[1:])]


@pytest.mark.parametrize("form", shapes.RECURRENCE, ids=lambda f: "x".join(map(str, f[0])))
def test_every_form(form):
    """Every number of units and wavefronts, sequences as they are, in parts and in order."""
    (count, mean, c, ragged), units = form[:2]
    offsets = [0]
    for n in lengths_of(count, mean, ragged):
        offsets.append(offsets[-1] + n)
    small = offsets[-1] * c < 1 << 21
    for kind in ("f32", "f16", "bf16") if small else ("bf16",):
        run(offsets, offsets[-1], c, kind, seed=mean, uniform=not ragged, starts_share=0.03)
    if small and units > 1:
        run(offsets, offsets[-1], c, "bf16", seed=mean, uniform=not ragged, starts_share=0.0, gap=1, at=1)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("c", [5, 66])
def test_long_sequences_in_parts(kind, c):
    """Few units over many steps: every sequence is cut into parts."""
    assert B.recurrence_workspace(4500, 3, c) > 0
    run([0, 4001, 4001, 4500], 4500, c, kind, seed=c, starts_share=0.003)
    run([0, 2100], 2100, c, kind, seed=c + 1, starts_share=0.0, spread=1.0)


@pytest.mark.parametrize("kind,gap,at", [("f32", 3, 1), ("f16", 1, 1), ("bf16", 5, 3), ("bf16", 0, 1), ("f16", 2, 0)])
def test_rows_apart_and_odd_addresses(kind, gap, at):
    run([0, 40, 41, 77], 77, 30, kind, gap=gap, at=at, seed=gap)
    run([0, 40, 41, 77], 77, 31, kind, gap=gap, at=at, seed=gap)


def test_without_states_and_starts():
    run([0, 50, 90], 90, 33, "f32", starts_share=0.0, with_first=False)
    run([0, 45, 90], 90, 33, "f32", starts_share=0.1, with_first=False)


@pytest.mark.parametrize("rows", [4, 3000])
def test_starts_end_what_was_before(rows):
    """An episode's start cuts states and gradients that are NaN or infinite."""
    c, cut = 6, rows // 2
    z, v, dy = torch.zeros(rows, c, device=DEV), torch.ones(rows, c, device=DEV), torch.ones(rows, c, device=DEV)
    v[cut - 1] = float("nan")
    v[cut - 2, 1] = float("inf")
    dy[cut] = 1.0
    dy[cut + 1, 2] = float("nan")
    starts = torch.zeros(rows, dtype=torch.uint8, device=DEV)
    starts[cut] = 7
    first = torch.full((1, c), float("nan"), device=DEV)
    starts[0] = 1
    y, dz, dv = (torch.empty(rows, c, device=DEV) for _ in range(3))
    last, dfirst = torch.empty(1, c, device=DEV), torch.empty(1, c, device=DEV)
    ws = torch.empty(max(16, B.recurrence_workspace(rows, 1, c)), dtype=torch.uint8, device=DEV)
    B.recurrence_forward(z, v, first, y, last, None, starts, ws)
    assert bool(torch.isfinite(y[:cut - 2]).all()) and bool(torch.isnan(y[cut - 1]).all())
    assert bool(torch.isfinite(y[cut:]).all()) and bool(torch.isfinite(last).all())
    assert bool((y[cut] == 0.5).all())
    B.recurrence_backward(dy, None, z, v, y, first, dz, dv, dfirst, None, starts, ws)
    assert bool(torch.isnan(dv[cut:cut + 2, 2]).all()) and bool(torch.isfinite(dv[:cut]).all()) and bool((dfirst == 0).all())


def test_gates_at_their_ends():
    """Gates of infinite and large z: everything kept, everything replaced."""
    inf = float("inf")
    z = torch.tensor([[inf, -inf, 200.0, -200.0, 0.0]], device=DEV)
    v, first = torch.full((1, 5), 3.0, device=DEV), torch.full((1, 5), 5.0, device=DEV)
    y, last = torch.empty(1, 5, device=DEV), torch.empty(1, 5, device=DEV)
    B.recurrence_forward(z, v, first, y, last)
    assert y.tolist() == [[5.0, 3.0, 5.0, 3.0, 4.0]] and bool((last == y).all())
    state = first.clone()
    B.recurrence_step(z, v, state, y)
    assert y.tolist() == [[5.0, 3.0, 5.0, 3.0, 4.0]] and bool((state == y).all())


def test_bad_offsets_stay_inside():
    """Offsets that lie outside of the rows, or fall, name no row that does not exist."""
    rows, c = 20, 8
    for values in ([-5, 10, 40], [30, 40, 50], [15, 5, 20], [-(1 << 31), (1 << 31) - 1, 3]):
        Z, V, Y = Framed(rows, c, torch.float32, 0, 0, 0.5), Framed(rows, c, torch.float32, 0, 0, 0.5), Framed(rows, c, torch.float32, 0, 0)
        last = torch.empty(2, c, device=DEV)
        B.recurrence_forward(Z.m, V.m, None, Y.m, last, torch.tensor(values, dtype=torch.int32, device=DEV))
        Y.get()
        DZ, DV = Framed(rows, c, torch.float32, 0, 0), Framed(rows, c, torch.float32, 0, 0)
        B.recurrence_backward(Y.m, None, Z.m, V.m, Y.m, None, DZ.m, DV.m, None, torch.tensor(values, dtype=torch.int32, device=DEV))
        DZ.get()
        DV.get()


def test_nothing_to_do():
    c = 8
    none = torch.empty(0, c, device=DEV)
    first, last = torch.randn(3, c, device=DEV), torch.zeros(3, c, device=DEV)
    B.recurrence_forward(none, none, first, none, last)
    assert bool((last == first).all())
    B.recurrence_backward(none, first, none, none, none, first, none, none, last)
    assert bool((last == first).all())
    rows = torch.zeros(4, c, device=DEV)
    y = torch.full((4, c), SENTINEL, device=DEV)
    B.recurrence_forward(rows, rows, None, y, None, torch.zeros(1, dtype=torch.int32, device=DEV))
    assert bool((y == SENTINEL).all())
    B.recurrence_step(none, none, none, none)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,c,gap,at", [(1, 1, 0, 0), (1, 256, 0, 0), (3, 77, 3, 1), (300, 1000, 0, 0), (16, 24, 1, 0)])
def test_step(kind, rows, c, gap, at):
    """Steps one after the other give what the sequence gives."""
    g = torch.Generator().manual_seed(rows + c)
    t = TYPES[kind]
    state = torch.randn(rows, c, generator=g)
    ref, bound = state.double(), torch.zeros(rows, c, dtype=torch.float64)
    d_state = state.to(DEV)
    a = ref.abs()
    for k in range(3):
        z, v = (torch.randn(rows, c, generator=g) * 2).to(t), torch.randn(rows, c, generator=g).to(t)
        starts = (torch.rand(rows, generator=g) < 0.3).to(torch.uint8) if k else None
        if k:
            ref, bound, a = (torch.where(starts[:, None] != 0, torch.zeros_like(x), x) for x in (ref, bound, a))
        Z, V, Y = Framed(rows, c, t, gap, at, z.to(DEV)), Framed(rows, c, t, gap, at, v.to(DEV)), Framed(rows, c, t, gap, at)
        B.recurrence_step(Z.m, V.m, d_state, Y.m if k < 2 else None, None if starts is None else starts.to(DEV))
        f, rest = torch.sigmoid(z.double()), torch.sigmoid(-z.double())
        ref, a = f * ref + rest * v.double(), f * a + rest * v.double().abs()
        bound = f * bound + ((1.5 * z.double().abs() + 6) * U + 4 * U) * a
        near(d_state.cpu().double(), ref, bound, "f32", "state")
        if k < 2:
            near(Y.get(), ref, bound, kind, "y")


def test_differences():
    """The gradients against differences of the forward pass: a sum over y and last with fixed weights, moved along one direction."""
    rows, c, n, h = 60, 6, 3, 2.0 ** -7
    g = torch.Generator().manual_seed(5)
    off = torch.tensor([0, 25, 25, 60], dtype=torch.int32, device=DEV)
    starts = (torch.rand(rows, generator=g) < 0.1).to(torch.uint8).to(DEV)
    z, v, dy, tz, tv = (torch.randn(rows, c, generator=g).to(DEV) for _ in range(5))
    first, dlast, tf = (torch.randn(n, c, generator=g).to(DEV) for _ in range(3))
    y, dz, dv = (torch.empty(rows, c, device=DEV) for _ in range(3))
    last, dfirst = torch.empty(n, c, device=DEV), torch.empty(n, c, device=DEV)

    def value(s):
        B.recurrence_forward(z + s * tz, v + s * tv, first + s * tf, y, last, off, starts)
        return float((y.double() * dy.double()).sum() + (last.double() * dlast.double()).sum())

    ends = [value(s * h) for s in (2, 1, -1, -2)]
    value(0.0)
    B.recurrence_backward(dy, dlast, z, v, y, first, dz, dv, dfirst, off, starts)
    slope = float((dz.double() * tz.double()).sum() + (dv.double() * tv.double()).sum() + (dfirst.double() * tf.double()).sum())
    want = (8 * (ends[1] - ends[2]) - (ends[0] - ends[3])) / (12 * h)
    # fp32 values of some 400 terms of size 1 each off by some 30 U, over h: 400 * 30 * 2^-24 / 2^-7 < 0.1; h^4 terms are below 1e-4 of it
    assert abs(slope - want) < 0.1 and abs(want) > 2.0


def test_captured_and_replayed():
    """A step and a sequence's passes, captured on a stream of their own and replayed between eager work."""
    rows, c = 3000, 10
    z, v, dy = (torch.randn(rows, c, device=DEV) for _ in range(3))
    state = torch.zeros(4, c, device=DEV)
    out = {k: torch.empty(rows, c, device=DEV) for k in ("y", "dz", "dv")}
    ys = torch.empty(4, c, device=DEV)
    ws = torch.empty(B.recurrence_workspace(rows, 1, c), dtype=torch.uint8, device=DEV)
    assert ws.numel()

    def work():
        B.recurrence_forward(z, v, None, out["y"], None, None, None, ws)
        B.recurrence_backward(dy, None, z, v, out["y"], None, out["dz"], out["dv"], None, None, None, ws)
        B.recurrence_step(z[:4], v[:4], state, ys)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work()
    for k in range(4):
        z.copy_(torch.randn(rows, c, device=DEV))
        state.zero_()
        work()
        torch.cuda.synchronize()
        want = {n: t.clone() for n, t in out.items()}, state.clone(), ys.clone()
        for t in out.values():
            t.fill_(SENTINEL)
        state.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((out[n] == want[0][n]).all()) for n in out) and bool((state == want[1]).all()) and bool((ys == want[2]).all()), k
