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
