"""The learner's operators at the ends of what they take."""
import pytest
import torch

from paper_1910_01055_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_products_of_a_billion_rows():
    """More rows than a launch has workgroups of 64; one value each, whose products are exact in 4 bits and in bfloat16."""
    rows, part = (1 << 30) + 77, 1 << 27
    values = torch.tensor([1.0, 1.5, -2.0, 3.0, 0.0, -6.0, 0.75], dtype=torch.bfloat16, device=DEV)
    x = torch.empty(rows, 1, dtype=torch.bfloat16, device=DEV)
    for at in range(0, rows, part):
        n = min(part, rows - at)
        x[at:at + n, 0] = values[(torch.arange(at, at + n, device=DEV) // 3) % 7]
    w = B.mx4_empty(1, 1)
    B.mx4_quantize(torch.full((1, 1), 1.5, device=DEV), w)
    y = torch.full((rows, 1), 77.0, dtype=torch.bfloat16, device=DEV)

    def check():
        for at in range(0, rows, part):
            assert torch.equal(y[at:at + part], x[at:at + part] * 1.5), at

    print("[input grad]", flush=True)
    size = B.mx4_input_grad_workspace(rows, 1, 1)
    B.mx4_input_grad(x, w, y, torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)
    check()
    y.fill_(77.0)
    print("[linear]", flush=True)
    B.mx4_linear(x, w, None, y, torch.empty(B.mx4_linear_workspace(rows, 1, 1), dtype=torch.uint8, device=DEV))
    check()


LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def test_every_scale():
    """Blocks of every scale, those among them that the conversions never make: 4-bit values from 2^128 on (scales 253 and 254) are
    infinities where they become numbers of their own, and are not in products of 4-bit tensors."""
    scales = torch.arange(256, dtype=torch.uint8)[:, None].contiguous()
    low, high = torch.arange(0, 32, 2) % 16, torch.arange(1, 32, 2) % 16
    codes = (low | high << 4).to(torch.uint8).expand(256, 16).contiguous()
    c = torch.arange(32) % 16
    w = LEVELS[c % 8] * torch.where(c >= 8, -1.0, 1.0) * torch.exp2(scales.double() - 127)
    w[255] = float("nan")
    steps = torch.randint(-127, 128, (256, 32), dtype=torch.int8, generator=torch.Generator().manual_seed(5))
    steps[:, :3] = torch.tensor([127, -127, 1], dtype=torch.int8)
    k = steps.double() * torch.exp2(scales.double() - 133)
    k[255] = float("nan")

    def same(got, want, what):
        got = got.cpu()
        want = want.to(torch.float32).to(got.dtype)
        assert torch.equal(torch.isnan(got), torch.isnan(want)), what
        assert torch.equal(got.nan_to_num(0.5, 7.0, -7.0), want.nan_to_num(0.5, 7.0, -7.0)), what

    q, kept = B.Mx4(codes.to(DEV), scales.to(DEV), 32), B.Ckpt8(steps.to(DEV), scales.to(DEV), 32)
    n = 253  # (of finite 4-bit values)
    some, some_kept = B.Mx4(q.codes[:n].contiguous(), q.scales[:n].contiguous(), 32), B.Ckpt8(kept.codes[:n].contiguous(), kept.scales[:n].contiguous(), 32)
    ws = torch.empty(max(16, B.mx4_input_grad_workspace(n, n, 32), B.ckpt8_weight_grad_workspace(n, n, 32)), dtype=torch.uint8, device=DEV)
    for t in (torch.float32, torch.float16, torch.bfloat16):
        out = torch.empty(256, 32, dtype=t, device=DEV)
        B.mx4_dequantize(q, out)
        same(out, w, "dequantize")
        B.ckpt8_unpack(kept, out)
        same(out, k, "unpack")
        one = torch.eye(n, dtype=t, device=DEV)
        B.mx4_input_grad(one, some, out[:n], ws)
        same(out[:n], w[:n], "input grad")
        dw = torch.empty(n, 32, device=DEV)
        B.ckpt8_weight_grad(one, some_kept, dw, None, ws)
        same(dw, k[:n], "weight grad")
    for scale in (100, 127, 140):  # one 1.0 of that scale to a row; few rows, and enough for tiles
        one = torch.zeros(32, 16, dtype=torch.uint8)
        one[torch.arange(32), torch.arange(32) // 2] = (2 << 4 * (torch.arange(32) % 2)).to(torch.uint8)
        for times in (1, 40):
            x = B.Mx4(one.repeat(times, 1).to(DEV), torch.full((32 * times, 1), scale, dtype=torch.uint8, device=DEV), 32)
            many = B.Mx4(q.codes.repeat(times, 1), q.scales.repeat(times, 1), 32)
            y = torch.empty(32 * times, 256 * times, device=DEV)
            B.mx4_matmul(x, many, None, y)
            same(y, (w.t() * 2.0 ** (scale - 127)).repeat(times, times), ("matmul", scale, times))


def test_pinned_memory():
    """Tensors that the host allocated for the GPU are tensors like others."""
    x = torch.randn(33, 70, generator=torch.Generator().manual_seed(3))
    pinned = torch.empty(33, 70, pin_memory=True).copy_(x)
    there, here = B.mx4_empty(33, 70), B.mx4_empty(33, 70)
    B.mx4_quantize(pinned, there)
    B.mx4_quantize(x.to(DEV), here)
    assert torch.equal(there.codes, here.codes) and torch.equal(there.scales, here.scales)
    with pytest.raises(ValueError):
        B.mx4_quantize(x, here)
