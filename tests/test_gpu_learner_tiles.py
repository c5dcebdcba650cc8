"""The learner's products on every tile that they may take (which learner_shapes.py lists), and LayerNorm's gradients over many rows: whole
numbers whose sums fp32 holds exactly, so that a term that is missing, foreign or counted twice shows."""
import math
import zlib

import learner_shapes as shapes
import pytest
import torch

from paper_1910_01055_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SENTINEL = 77.0
EXACT = 2 ** 24  # whole numbers up to here are fp32's


def generator(*key):
    return torch.Generator(device=DEV).manual_seed(zlib.crc32(repr(key).encode()))


def pick(g, values, *shape):
    v = torch.tensor(values, dtype=torch.float64, device=DEV)
    return v[torch.randint(len(values), shape, generator=g, device=DEV)]


def framed(rows, cols, dtype, gap=0, first=0, values=None):
    """A matrix whose rows lie `gap` apart and start at element `first`, and a check that nothing around it was written."""
    ld = cols + gap
    buf = torch.full((first + rows * ld + 64,), SENTINEL, dtype=dtype, device=DEV)
    m = buf[first:first + rows * ld].view(rows, ld)[:, :cols]
    if values is not None:
        m.copy_(values)

    def check():
        around = buf.clone()
        around[first:first + rows * ld].view(rows, ld)[:, :cols] = SENTINEL
        assert bool((around == SENTINEL).all()), "values outside of the matrix were written"
    return m, check


def scratch(size):
    return torch.full((size,), 255, dtype=torch.uint8, device=DEV) if size else None


def ckpt(x):
    kept = B.ckpt8_empty(*x.shape)
    B.ckpt8_pack(x, kept)
    return kept


def mx4(x):
    q = B.mx4_empty(*x.shape)
    B.mx4_quantize(x.float(), q)
    return q


def wide_numbers(g, kind, rows, cols):
    """dy: small whole numbers, and now and then one that takes all bits of its type (24, 11 or 8, in fp32 all three parts of it)."""
    dy = pick(g, [-3, -2, -1, 0, 1, 2, 3], rows, cols)
    top = {"f32": 2.0 ** 20 - 1, "f16": 2.0 ** 11 - 1, "bf16": 2.0 ** 8 - 1}[kind]
    some = torch.arange(rows, device=DEV)[:, None] * 31 + torch.arange(cols, device=DEV) * 17
    return torch.where(some % 499 == 0, torch.full_like(dy, top), dy)


def product(a, b):
    """a b and the sum of its terms' magnitudes, in fp64."""
    return a @ b, (a.abs() @ b.abs()).max().item()


SMALL = [-1, 0, 0, 1]  # so that sums of many large numbers stay exact


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", [s[0] for s in shapes.WEIGHT_GRAD], ids=str)
def test_weight_grad(sizes, kind):
    print(f"[weight grad] {sizes} {kind}", flush=True)
    rows, n, k = sizes
    g = generator("wg", sizes, kind)
    x, dy = pick(g, SMALL, rows, k), wide_numbers(g, kind, rows, n)
    want, most = product(dy.t().contiguous(), x)
    assert max(most, dy.abs().sum(0).max().item()) < EXACT
    kept, ws = ckpt(x.to(TYPES[kind])), scratch(B.ckpt8_weight_grad_workspace(rows, n, k))
    for gap, first in ((0, 0), (1, 1), (7, 0)):
        d, _ = framed(rows, n, TYPES[kind], gap, first, dy)
        dw, check = framed(n, k, torch.float32, gap, first)
        db, check_db = framed(1, n, torch.float32, 0, first)
        B.ckpt8_weight_grad(d, kept, dw, db[0], ws)
        check()
        check_db()
        assert torch.equal(dw.double(), want) and torch.equal(db[0].double(), dy.sum(0))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", [s[0] for s in shapes.INPUT_GRAD], ids=str)
def test_input_grad(sizes, kind):
    print(f"[input grad] {sizes} {kind}", flush=True)
    rows, n, k = sizes
    g = generator("ig", sizes, kind)
    w, dy = pick(g, SMALL, n, k), wide_numbers(g, kind, rows, n)
    want, most = product(dy, w)
    assert most < EXACT
    q, ws = mx4(w), scratch(B.mx4_input_grad_workspace(rows, n, k))
    for gap, first in ((0, 0), (1, 1), (8, 0)):
        d, _ = framed(rows, n, TYPES[kind], gap, first, dy)
        dx, check = framed(rows, k, TYPES[kind], gap, first)
        B.mx4_input_grad(d, q, dx, ws)
        check()
        assert torch.equal(dx, want.to(TYPES[kind]))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", [s[0] for s in shapes.MX4], ids=str)
def test_mx4_products(sizes, kind):
    print(f"[mx4] {sizes} {kind}", flush=True)
    rows, n, k = sizes
    g = generator("mx4", sizes, kind)
    values = [-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6]
    x, w, bias = pick(g, values, rows, k), pick(g, values, n, k), pick(g, [-40, -7, 0, 1, 100], n)
    # rows and features of scales of their own: a scale that is read from another row or block shows
    ex, ew = torch.exp2(torch.arange(rows, device=DEV).double() % 3)[:, None], torch.exp2(torch.arange(n, device=DEV).double() % 4)[:, None]
    blocks = torch.exp2((torch.arange(k, device=DEV) // 32).double() % 5 - 2)  # x's up, w's down: the products stay whole
    w = w * ew / blocks
    x = x * ex * blocks
    want, most = product(x, w.t().contiguous())
    want = want + bias
    assert most + 100 < EXACT
    xq, wq = mx4(x), mx4(w)
    back = torch.empty(n, k, device=DEV)
    B.mx4_dequantize(wq, back)
    assert torch.equal(back.double(), w)  # as the test is meant
    for gap, first in ((0, 0), (3, 1)):
        y, check = framed(rows, n, TYPES[kind], gap, first)
        B.mx4_matmul(xq, wq, bias.float(), y)
        check()
        assert torch.equal(y, want.to(TYPES[kind]))
        z, check = framed(rows, n, TYPES[kind], gap, first)
        B.mx4_linear(framed(rows, k, TYPES[kind], gap, first, x)[0], wq, bias.float(), z, scratch(B.mx4_linear_workspace(rows, n, k)))
        check()
        assert torch.equal(z, y)


@pytest.mark.parametrize("sizes", [(1009, 1111, 1009), (2051, 2100, 1100), (4101, 4099, 777)], ids=str)
def test_mx4_tiles_of_what_is_not_finite(sizes):
    """A NaN or an infinity in any block, the last and short one among them, and only in its row's and its feature's results."""
    rows, n, k = sizes
    g = generator("nan", sizes)
    x, w = torch.randn(rows, k, generator=g, device=DEV), torch.randn(n, k, generator=g, device=DEV)
    bad_x, bad_w = torch.tensor([0, 65, rows - 1], device=DEV), torch.tensor([3, 130, n - 1], device=DEV)
    x[bad_x, torch.tensor([5, k // 2, k - 1], device=DEV)] = torch.tensor([math.nan, math.inf, -math.inf], device=DEV)
    w[bad_w, torch.tensor([k - 1, 40, k - 2], device=DEV)] = torch.tensor([math.inf, math.nan, math.nan], device=DEV)
    bad = torch.zeros(rows, n, dtype=torch.bool, device=DEV)
    bad[bad_x], bad[:, bad_w] = True, True
    y = torch.empty(rows, n, device=DEV)
    B.mx4_matmul(mx4(x), mx4(w), None, y)
    assert torch.equal(torch.isnan(y), bad) and bool(torch.isfinite(y[~bad]).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", [(71, 205, 99), (1681, 301, 300), (2041, 1101, 2052)], ids=str)
def test_input_grad_of_weights_at_the_ends(sizes, kind):
    """4-bit weights of the smallest scales, whose values are denormal in bfloat16 too, of the largest and of NaNs."""
    rows, n, k = sizes
    g = generator("ends", sizes, kind)
    w = pick(g, [-6, -4, -3, -2, -1, 1, 2, 3, 4, 6], n, k)
    columns = torch.arange(k, device=DEV) // 32
    scale = torch.full((k,), 1.0, dtype=torch.float64, device=DEV)
    scale[columns == 0] = 2.0 ** -128  # (6 steps of the smallest scale's half: its elements 0.5 .. 3)
    scale[columns == 1] = 2.0 ** 125
    w = w * scale
    q = mx4(w)
    back = torch.empty(n, k, device=DEV)
    B.mx4_dequantize(q, back)
    assert torch.equal(back.double(), w) and int(q.scales[:, 0].max()) == 0 and int(q.scales[:, 1].min()) == 252
    q.scales[7, 2] = 255
    dy = torch.zeros(rows, n, dtype=torch.float64, device=DEV)
    dy[torch.arange(rows, device=DEV), torch.arange(rows, device=DEV) % n] = 1.0  # one weight each: nothing overflows
    want = dy @ w
    dx = torch.empty(rows, k, dtype=TYPES[kind], device=DEV)
    B.mx4_input_grad(dy.to(TYPES[kind]), q, dx, scratch(B.mx4_input_grad_workspace(rows, n, k)))
    of_nan = (columns == 2).expand(rows, k)  # 0 times a NaN is one
    assert torch.equal(torch.isnan(dx), of_nan)
    assert torch.equal(dx[~of_nan], want.to(torch.float32).to(TYPES[kind])[~of_nan])


FAR = 1 << 21  # the largest distance between rows


def far(rows, cols, dtype):
    return torch.empty(rows * FAR, dtype=dtype, device=DEV).view(rows, FAR)[:, 3:3 + cols]


@pytest.mark.parametrize("sizes", [(203, 4431, 655), (201, 1517, 5457)], ids=str)
def test_weight_grad_of_rows_far_apart(sizes):
    """On tiles of 128 and 256 in one slice: windows that hold some dozen rows move on."""
    rows, n, k = sizes
    g = generator("far", sizes)
    x, dy = pick(g, SMALL, rows, k), wide_numbers(g, "f32", rows, n)
    d = far(rows, n, torch.float32)
    d.copy_(dy)
    dw, db = torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    B.ckpt8_weight_grad(d, ckpt(x.float()), dw, db, scratch(B.ckpt8_weight_grad_workspace(rows, n, k)))
    assert torch.equal(dw.double(), dy.t().contiguous() @ x) and torch.equal(db.double(), dy.sum(0))


@pytest.mark.parametrize("sizes", [(1681, 5669, 77), (131, 4797, 3305)], ids=str)
def test_input_grad_of_rows_far_apart(sizes):
    """On tiles of 128 and 256: the rows of a tile lie as far as a window shows, and so do those of the result."""
    rows, n, k = sizes
    g = generator("far", sizes)
    w, dy = pick(g, SMALL, n, k), wide_numbers(g, "f32", rows, n)
    d, dx = far(rows, n, torch.float32), far(rows, k, torch.float32)
    d.copy_(dy)
    B.mx4_input_grad(d, mx4(w), dx, scratch(B.mx4_input_grad_workspace(rows, n, k)))
    assert torch.equal(dx.double(), dy @ w)


def test_mx4_product_to_rows_far_apart():
    rows, n, k = 2051, 2100, 300
    g = generator("far mx4")
    x, w = pick(g, SMALL, rows, k), pick(g, SMALL, n, k)
    y = far(rows, n, torch.float32)
    B.mx4_matmul(mx4(x), mx4(w), None, y)
    assert torch.equal(y.double(), x @ w.t().contiguous())


# ---- LayerNorm's gradients.  With a mean of 0 and a reciprocal deviation of 1, h is x itself, and dgamma and dbeta are sums of whole numbers.

@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 8), (511, 64), (16500, 301), (4099, 1024), (2100, 1501), (1100, 5003), (600, 8205), (301, 16384), (1_300_003, 20)])
def test_layernorm_gradients_of_whole_numbers(rows, cols, kind):
    print(f"[layernorm] {rows}x{cols} {kind}", flush=True)
    g = generator("ln", rows, cols, kind)
    x, dy = pick(g, [-3, -2, -1, 0, 1, 2, 3], rows, cols), pick(g, [-2, -1, 0, 1, 2], rows, cols)
    gamma = pick(g, [1, 2], cols)
    assert 6 * rows < EXACT
    X, D = x.to(TYPES[kind]), dy.to(TYPES[kind])
    mean, rstd = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    gd = dy * gamma
    dx_want = gd - gd.mean(1, keepdim=True) - x * (gd * x).mean(1, keepdim=True)
    ws = scratch(B.layernorm_backward_workspace(rows, cols))
    for src in (X, ckpt(X)):
        dx, check = framed(rows, cols, TYPES[kind], 3, 1)
        dgamma, dbeta = torch.full((cols,), SENTINEL, device=DEV), torch.full((cols,), SENTINEL, device=DEV)
        B.layernorm_backward(D, src, gamma.float(), mean, rstd, dx, dgamma, dbeta, ws)
        check()
        assert torch.equal(dgamma.double(), (dy * x).sum(0)) and torch.equal(dbeta.double(), dy.sum(0))
        # The row's sums are exact.  With |g|, |c1| <= 4, |h| <= 3 and |c2| <= 12 the rest is off, in units of 2^-24 at most, by 4 (c1), 8
        # (g - c1), 36 (c2, times h), 36 (the product) and 48 (the difference)
        off = 132 * 2.0 ** -24
        out = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[kind]
        assert bool(((dx.double() - dx_want).abs() <= off + out * (dx_want.abs() + off)).all())
