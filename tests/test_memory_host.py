"""What gated layers, the recurrence and the optimizer refuse, and the sizes they ask for (no GPU work: refused calls return before any)."""
import ctypes as C
import math

import pytest
import torch

from paper_1910_01055_amd import binding as B
from test_learner_binding import Library, Pinned
from test_learner_host import BAD_MATRICES, V, WS, mat

BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return B.load()


def size_of(fn, *args):
    n = C.c_uint64(77)
    status = fn(*args, C.byref(n))
    return status, n.value


# ---- gated layers: x [4][32], weights [24][32], y, gate and up [4][24]
def gated_forward(lib, x=None, wg=None, wu=None, y=None, gate=None, up=None, act=1, ws=WS, size=BIG):
    x, wg, wu, y, gate, up = (mat(*s) if m is None else m for m, s in zip((x, wg, wu, y, gate, up), ((4, 32), (24, 32), (24, 32), (4, 24), (4, 24), (4, 24))))
    return lib.aq_gated_forward(x, wg, wu, act, y, None if gate == "no" else gate, None if up == "no" else up, ws, size, None)


def gated_backward(lib, act=1, ws=WS, size=BIG, **other):
    shapes = {"dy": (4, 24), "x": (4, 32), "wg": (24, 32), "wu": (24, 32), "gate": (4, 24), "up": (4, 24), "dx": (4, 32), "dwg": (24, 32), "dwu": (24, 32)}
    m = [other.get(k, mat(*s)) for k, s in shapes.items()]
    return lib.aq_gated_backward(*m[:6], act, *m[6:], ws, size, None)


def test_gated_matrices(lib):
    for bad, want in BAD_MATRICES:
        for name in ("x", "wg", "wu", "y"):
            if bad is not None:
                assert gated_forward(lib, **{name: bad}) in (want, B.ESHAPE), name
        for name in ("dy", "x", "wg", "wu", "gate", "up"):
            assert gated_backward(lib, **{name: bad}) in (want, B.ESHAPE), name
    E = B.ESHAPE
    for name, other in (("wg", (24, 31)), ("wu", (23, 32)), ("wu", (24, 33)), ("y", (5, 24)), ("y", (4, 23)), ("gate", (4, 25)), ("up", (3, 24)), ("x", (4, 33))):
        assert gated_forward(lib, **{name: mat(*other)}) == E, name
    for name, other in (("dy", (4, 25)), ("dy", (5, 24)), ("x", (4, 31)), ("wg", (24, 33)), ("wu", (25, 32)), ("gate", (4, 23)), ("up", (5, 24)), ("dx", (4, 33)),
                        ("dx", (5, 32)), ("dwg", (23, 32)), ("dwu", (24, 31))):
        assert gated_backward(lib, **{name: mat(*other)}) == E, name
    for name, shape in (("wg", (24, 32)), ("wu", (24, 32)), ("y", (4, 24)), ("gate", (4, 24)), ("up", (4, 24))):
        assert gated_forward(lib, **{name: mat(*shape, dtype=2)}) == E
    for name, shape in (("dy", (4, 24)), ("wg", (24, 32)), ("gate", (4, 24)), ("dx", (4, 32)), ("dwu", (24, 32))):
        assert gated_backward(lib, **{name: mat(*shape, dtype=1)}) == E
    for act in (-1, 4):
        assert gated_forward(lib, act=act) == B.EINVAL and gated_backward(lib, act=act) == B.EINVAL
    assert gated_forward(lib, gate="no") == B.EINVAL and gated_forward(lib, up="no") == B.EINVAL
    assert gated_backward(lib, dwg=None) == B.EINVAL and gated_backward(lib, dwu=None) == B.EINVAL


def test_gated_workspace(lib):
    for fn in (lib.aq_gated_forward_workspace, lib.aq_gated_backward_workspace):
        assert fn(4, 24, 32, 0, None) == B.EINVAL
        for args, want in (((-1, 24, 32, 0), B.EINVAL), ((4, -1, 32, 0), B.EINVAL), ((4, 24, -2, 0), B.EINVAL), ((4, 24, 32, 3), B.EINVAL), ((4, 0, 32, 0), B.ESHAPE),
                           ((4, 24, 0, 0), B.ESHAPE), ((4, (1 << 20) + 1, 32, 0), B.ESHAPE), ((1 << 31, 24, 32, 0), B.ESHAPE), ((1 << 28, 64, 8, 0), B.ESHAPE)):
            assert size_of(fn, *args) == (want, 77)
    # few rows need none; others theirs, and no less
    assert size_of(lib.aq_gated_forward_workspace, 4, 24, 32, 0) == (B.OK, 0)
    for dtype in (0, 2):
        status, need = size_of(lib.aq_gated_forward_workspace, 100, 24, 32, dtype)
        big = {"x": mat(100, 32, dtype), "wg": mat(24, 32, dtype), "wu": mat(24, 32, dtype), "y": mat(100, 24, dtype), "gate": mat(100, 24, dtype), "up": mat(100, 24, dtype)}
        assert need > 0 and gated_forward(lib, size=need - 1, **big) == B.EINVAL and gated_forward(lib, ws=WS + 8, **big) == B.EINVAL
        assert gated_forward(lib, ws=None, **big) == B.EINVAL
    status, need = size_of(lib.aq_gated_backward_workspace, 4, 24, 32, 0)
    assert need > 0 and gated_backward(lib, size=need - 1) == B.EINVAL and gated_backward(lib, ws=None) == B.EINVAL


# ---- the recurrence: 6 rows of 8 units, 2 sequences
def forward(lib, z=None, v=None, y=None, off=V, count=2, starts=None, first=V, last=2 * V, ws=WS, size=BIG):
    z, v, y = (mat(6, 8) if m is None else m for m in (z, v, y))
    return lib.aq_recurrence_forward(z, v, off, count, starts, first, y, last, ws, size, None)


def backward(lib, off=V, count=2, starts=None, first=V, dlast=2 * V, dfirst=3 * V, ws=WS, size=BIG, **other):
    m = [other.get(k, mat(6, 8)) for k in ("dy", "z", "v", "y", "dz", "dv")]
    return lib.aq_recurrence_backward(m[0], dlast, m[1], m[2], m[3], off, count, starts, first, m[4], m[5], dfirst, ws, size, None)


def test_recurrence(lib):
    for bad, want in BAD_MATRICES:
        if bad is not None:
            for name in ("z", "v", "y"):
                assert forward(lib, **{name: bad}) in (want, B.ESHAPE)
            assert lib.aq_recurrence_step(mat(6, 8), bad, None, V, mat(6, 8), None) in (want, B.ESHAPE)
        for name in ("dy", "z", "v", "y", "dz", "dv"):
            assert backward(lib, **{name: bad}) in (want, B.ESHAPE)
    for other in (mat(5, 8), mat(6, 7), mat(6, 8, 2)):
        assert forward(lib, v=other) == B.ESHAPE and forward(lib, y=other) == B.ESHAPE
        for name in ("dy", "v", "y", "dz", "dv"):
            assert backward(lib, **{name: other}) == B.ESHAPE
        assert lib.aq_recurrence_step(mat(6, 8), other, None, V, None, None) == B.ESHAPE
        assert lib.aq_recurrence_step(mat(6, 8), mat(6, 8), None, V, other, None) == B.ESHAPE
    for call in (forward, backward):
        assert call(lib, count=-1) == B.EINVAL and call(lib, off=V + 2) == B.EINVAL and call(lib, first=V + 1) == B.EINVAL
        assert call(lib, off=None, count=4) == B.ESHAPE  # six rows are no four equal parts
        assert call(lib, count=1 << 31) == B.ESHAPE and call(lib, count=(1 << 25) + 1) == B.ESHAPE
    # states in place would be read behind their own writing where a sequence is in parts
    assert forward(lib, first=V, last=V) == B.EINVAL
    assert backward(lib, dlast=V, dfirst=V) == B.EINVAL and backward(lib, first=V, dfirst=V) == B.EINVAL
    assert forward(lib, last=V + 2) == B.EINVAL and backward(lib, dlast=V + 3) == B.EINVAL and backward(lib, dfirst=V + 1) == B.EINVAL
    assert lib.aq_recurrence_step(mat(6, 8), mat(6, 8), None, None, None, None) == B.EINVAL
    assert lib.aq_recurrence_step(mat(6, 8), mat(6, 8), None, V + 1, None, None) == B.EINVAL
    for args, want in (((-1, 2, 8), B.EINVAL), ((6, -1, 8), B.EINVAL), ((6, 2, -8), B.EINVAL), ((6, 2, 0), B.ESHAPE), ((6, 1 << 31, 8), B.ESHAPE),
                       ((1 << 31, 2, 8), B.ESHAPE), ((6, 1 << 20, 257), B.ESHAPE)):
        assert size_of(lib.aq_recurrence_workspace, *args) == (want, 77)
    assert lib.aq_recurrence_workspace(6, 2, 8, None) == B.EINVAL
    assert size_of(lib.aq_recurrence_workspace, 6, 2, 8) == (B.OK, 0) and size_of(lib.aq_recurrence_workspace, 6, 0, 8) == (B.OK, 0)
    status, need = size_of(lib.aq_recurrence_workspace, 4096, 2, 8)
    long = {k: mat(4096, 8) for k in ("z", "v", "y")}
    assert need > 0 and forward(lib, size=need - 1, **long) == B.EINVAL and forward(lib, ws=None, **long) == B.EINVAL and forward(lib, ws=WS + 4, **long) == B.EINVAL


# ---- the optimizer
GOOD = dict(d_w=V, d_g=2 * V, d_m=3 * V, d_v=4 * V, d_m_scales=None, d_v_scales=None, d_copy=None, n=40, g_dtype=0, copy_dtype=0, moment_bits=32, decay=1)
HOW = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=1.0, step=1, d_lr=None, d_step=None, d_norm=None)
EIGHT = dict(moment_bits=8, d_m_scales=5 * V, d_v_scales=6 * V)


def tensors(**change):
    return (B.AqLearned * 2)(B.AqLearned(**GOOD), B.AqLearned(**{**GOOD, **change}))


def adamw(lib, how=None, **change):
    return lib.aq_adamw_step(tensors(**change), 2, C.byref(B.AqAdamw(**{**HOW, **(how or {})})), None)


BAD_TENSORS = [dict(n=-1), dict(d_m=None), dict(d_v=None), dict(d_m=3 * V + 2), dict(d_v=4 * V + 1), dict(moment_bits=16), dict(moment_bits=0),
               {**EIGHT, "d_m_scales": None}, {**EIGHT, "d_v_scales": None}, {**EIGHT, "d_m": 3 * V + 8}, {**EIGHT, "d_v": 4 * V + 1}]
BAD_GRADIENTS = [dict(d_g=None), dict(g_dtype=3), dict(g_dtype=-1), dict(d_g=2 * V + 2), dict(d_g=2 * V + 1, g_dtype=2)]


def test_structures_are_laid_out_as_in_the_header():
    assert C.sizeof(B.AqLearned) == 7 * 8 + 8 + 4 * 4
    assert C.sizeof(B.AqAdamw) == 6 * 8 + 8 + 3 * 8 == len(B._pack_adamw(*([0.0] * 6), 1, 0, 0, 0))


def test_optimizer(lib):
    for bad in BAD_TENSORS + BAD_GRADIENTS + [dict(d_w=None), dict(d_w=V + 2), dict(d_copy=7 * V, copy_dtype=0), dict(d_copy=7 * V + 1, copy_dtype=2)]:
        assert adamw(lib, **bad) == B.EINVAL, bad
    assert adamw(lib, n=(1 << 34) + 1) == B.ESHAPE
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=math.nan), dict(beta2=1.0), dict(beta2=-1.0), dict(eps=-1e-8), dict(eps=math.nan), dict(weight_decay=-1.0),
                dict(max_norm=0.0), dict(max_norm=math.nan), dict(lr=-1.0), dict(lr=math.nan), dict(step=0), dict(step=-3), dict(d_lr=V + 2), dict(d_step=V + 4),
                dict(d_norm=V + 1)):
        assert adamw(lib, bad) == B.EINVAL, bad
    how = C.byref(B.AqAdamw(**HOW))
    assert lib.aq_adamw_step(None, 2, how, None) == B.EINVAL and lib.aq_adamw_step(tensors(), -1, how, None) == B.EINVAL
    assert lib.aq_adamw_step(tensors(), 2, None, None) == B.EINVAL and lib.aq_adamw_step(tensors(), (1 << 20) + 1, how, None) == B.ESHAPE
    assert lib.aq_adamw_step(None, 0, how, None) == B.OK


def test_norm_and_conversion(lib):
    need = C.c_uint64(0)
    assert lib.aq_grad_norm_workspace(tensors(), 2, C.byref(need)) == B.OK and need.value > 0
    assert lib.aq_grad_norm_workspace(tensors(), 2, None) == B.EINVAL and lib.aq_grad_norm_workspace(tensors(n=-1), 2, C.byref(need)) == B.EINVAL
    for bad in BAD_GRADIENTS:
        assert lib.aq_grad_norm(tensors(**bad), 2, V, WS, BIG, None) == B.EINVAL, bad
    for norm, ws, size in ((None, WS, BIG), (V + 2, WS, BIG), (V, WS, need.value - 1), (V, None, BIG), (V, WS + 8, BIG)):
        assert lib.aq_grad_norm(tensors(), 2, norm, ws, size, None) == B.EINVAL
    for bad in BAD_TENSORS:
        assert lib.aq_moments_convert(tensors(**bad), tensors(), 2, None) == B.EINVAL
        assert lib.aq_moments_convert(tensors(), tensors(**bad), 2, None) == B.EINVAL
    assert lib.aq_moments_convert(tensors(), tensors(n=41), 2, None) == B.ESHAPE


# ---- the binding, on a library that takes every call
def stand_in(monkeypatch, device=-1):
    library = Library()
    monkeypatch.setattr(B, "_lib", library)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    monkeypatch.setattr(B, "_device", lambda: device)
    return library


def learned(n=70, bits=32, copy=None, device="cpu"):
    m = (lambda: torch.zeros(n, device=device)) if bits == 32 else lambda: B.moment8_zeros(n, device)
    return B.Learned(torch.zeros(n), torch.zeros(n), m(), m(), copy)


def calls(make):
    """Every call with the tensors that `make` gives for (name, *shape), by the names of its tensors."""
    f, u8, i32, i64 = torch.float32, torch.uint8, torch.int32, torch.int64
    t = {n: (lambda n=n, s=s, d=d: make(n, *s, dtype=d)) for n, s, d in (
        ("x", (4, 32), f), ("wg", (24, 32), f), ("wu", (24, 32), f), ("y", (4, 24), f), ("gate", (4, 24), f), ("up", (4, 24), f), ("dy", (4, 24), f),
        ("dx", (4, 32), f), ("dwg", (24, 32), f), ("dwu", (24, 32), f), ("ws", (64,), u8), ("z", (6, 8), f), ("v", (6, 8), f), ("h", (6, 8), f), ("dz", (6, 8), f),
        ("dv", (6, 8), f), ("first", (2, 8), f), ("last", (2, 8), f), ("dlast", (2, 8), f), ("dfirst", (2, 8), f), ("offsets", (3,), i32), ("starts", (6,), u8),
        ("state", (6, 8), f), ("norm", (1,), f), ("lr", (1,), f), ("step", (1,), i64))}
    g = lambda names: [t[n]() for n in names.split()]  # noqa: E731

    def gf(names="x wg wu y gate up ws"):
        a = g(names)
        B.gated_forward(a[0], a[1], a[2], "silu", a[3], a[4], a[5], a[6])

    def gb(names="dy x wg wu gate up dx dwg dwu ws"):
        a = g(names)
        B.gated_backward(*a[:6], "silu", *a[6:])

    def rf(names="z v first h last offsets starts ws"):
        B.recurrence_forward(*g(names))

    def rb(names="h dlast z v h first dz dv dfirst offsets starts ws"):
        B.recurrence_backward(*g(names))

    def rs(names="z v state h starts"):
        B.recurrence_step(*g(names))

    def aw(names="norm lr step"):
        norm, lr, step = g(names)
        B.adamw_step(B.LearnedSet([]), lr, 0.9, 0.99, 1e-8, 0.0, step, norm, 1.0)

    def gn(names="norm ws"):
        B.grad_norm(B.LearnedSet([]), *g(names))

    return {f: f.__defaults__[0].split() for f in (gf, gb, rf, rb, rs, aw, gn)}


def test_tensors_in_host_memory_and_of_other_devices_are_refused(monkeypatch):
    """Each tensor of each call in turn: ordinary host memory faults the GPU, and another device's tensors are not this stream's.  Pinned
    memory is taken."""
    library = stand_in(monkeypatch, device=3)

    class Here(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 3

    class Elsewhere(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 2

    def maker(kind, which=None, other=None):
        return lambda name, *shape, dtype: torch.zeros(shape, dtype=dtype).as_subclass(other if name == which else kind)

    for fn in calls(maker(Here)):
        fn()
        assert len(library.calls) == 1 and library.calls.pop()
    for fn in calls(maker(Pinned)):
        fn()
        assert len(library.calls) == 1 and library.calls.pop()
    names = {n for reads in calls(maker(Here)).values() for n in reads}
    for name in sorted(names):
        for other, what in ((torch.Tensor, "host memory"), (Elsewhere, "device 2")):
            refused = 0
            for fn, reads in calls(maker(Here, name, other)).items():
                if name in reads:
                    refused += 1
                    with pytest.raises(ValueError, match=what):
                        fn()
                    assert not library.calls, (name, fn.__name__)
            assert refused


def test_sets_of_tensors_are_refused(monkeypatch):
    library = stand_in(monkeypatch, device=3)
    on_host = B.LearnedSet([learned()])
    for call in (lambda: B.adamw_step(on_host, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1), lambda: B.grad_norm(on_host, torch.zeros(1).as_subclass(Pinned)),
                 lambda: B.moments_convert(on_host, on_host)):
        with pytest.raises(ValueError, match="host memory"):
            call()
        assert not library.calls
    with pytest.raises(ValueError):
        B.moments_convert(on_host, B.LearnedSet([]))


def test_shapes_and_types_are_refused(monkeypatch):
    library = stand_in(monkeypatch)
    z = torch.zeros(6, 8)
    states = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        B.recurrence_forward(z, z, states, z, None, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        B.recurrence_forward(z, z, states, z, None, torch.zeros(4, dtype=torch.int32))  # three sequences, two states
    with pytest.raises(ValueError):
        B.recurrence_forward(z, z, states, z, torch.zeros(3, 8))
    with pytest.raises(ValueError):
        B.recurrence_forward(z, z, states, z, None, None, torch.zeros(5, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.recurrence_forward(z, z, states, z, None, None, torch.zeros(6, dtype=torch.bool))
    with pytest.raises(ValueError):
        B.recurrence_forward(z, z, None, z, None, torch.zeros(0, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.recurrence_step(z, z, torch.zeros(6, 8, dtype=torch.float16))
    with pytest.raises(ValueError):
        B.recurrence_step(z, z, torch.zeros(8, 6).t())
    with pytest.raises(KeyError):
        B.gated_forward(z, z, z, "tanh", torch.zeros(6, 6))
    with pytest.raises(ValueError):
        B.adamw_step(B.LearnedSet([]), torch.zeros(2), 0.9, 0.99, 1e-8, 0.0, 1)
    with pytest.raises(ValueError):
        B.adamw_step(B.LearnedSet([]), 1e-3, 0.9, 0.99, 1e-8, 0.0, torch.zeros(1, dtype=torch.int32))
    assert not library.calls


def test_learned_tensors():
    f, w = torch.zeros(70), torch.zeros(7, 10)
    for bad in ((w.t(), f, f, f), (w.half(), f, f, f), (f, torch.zeros(71), f, f), (f, torch.zeros(70, dtype=torch.float64), f, f), (f, f, torch.zeros(70).half(), f),
                (f, f, f, torch.zeros(69)), (f, f, B.moment8_zeros(70, "cpu"), f), (f, f, f, B.moment8_zeros(70, "cpu")),
                (f, f, B.moment8_zeros(70, "cpu"), B.moment8_zeros(71, "cpu")), (f, f, f, f, torch.zeros(70)), (f, f, f, f, torch.zeros(71).half())):
        with pytest.raises(ValueError):
            B.Learned(*bad)
    codes, scales = torch.zeros(96, dtype=torch.uint8), torch.zeros(3, dtype=torch.uint8)
    B.Moment8(codes, scales, 70)
    odd = torch.zeros(100, dtype=torch.uint8)[1:97]
    for bad in ((codes, scales, 64), (codes, scales, 97), (codes[:64], scales, 70), (odd, scales, 70), (codes.to(torch.int8), scales, 70)):
        with pytest.raises(ValueError):
            B.Moment8(*bad)


def test_tensors_of_a_set_do_not_overlap():
    def parts(*views):
        return B.Learned(*views)

    new = lambda n=64: torch.zeros(n)  # noqa: E731
    one = learned()
    with pytest.raises(ValueError):
        B.LearnedSet([one, one])
    flat = torch.zeros(128)
    B.LearnedSet([parts(flat[:64], new(), new(), new()), parts(flat[64:], new(), new(), new())])
    for a, b in (((flat[:64], new(), new(), new()), (flat[63:127], new(), new(), new())), ((flat[:64], flat[:64], new(), new()), ()),
                 ((new(), new(), flat[:64], flat[32:96]), ()), ((flat[:64], new(), new(), new()), (new(), flat[10:74], new(), new()))):
        with pytest.raises(ValueError, match="overlap"):
            B.LearnedSet([parts(*p) for p in (a, b) if p])
    shared = new()  # a gradient that two tensors have is only read
    B.LearnedSet([parts(new(), shared, new(), new()), parts(new(), shared, new(), new())])
    m, v = B.moment8_zeros(64, "cpu"), B.moment8_zeros(64, "cpu")
    with pytest.raises(ValueError, match="overlap"):
        B.LearnedSet([B.Learned(new(), new(), m, m)])
    B.LearnedSet([B.Learned(new(), new(), m, v)])
