"""What the binding refuses of the learner's operators before a call reaches the library (no GPU work: the library is a stand-in that
takes every call)."""
import pytest
import torch

from paper_1910_01055_amd import binding as B


class Library:
    """Answers AQ_OK to everything."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or B.OK


@pytest.fixture
def lib(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "load", lambda: library)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    return library


def blocks(make, rows, cols):
    return make(rows, cols, device="cpu")


ROWS, N, K = 4, 40, 70


def operands():
    """x [rows][k], y and dy [rows][n], a checkpoint and 4-bit values of x, 4-bit weights [n][k] and what is laid out like them."""
    x, y = torch.zeros(ROWS, K), torch.zeros(ROWS, N)
    return (x, y, blocks(B.ckpt8_empty, ROWS, K), blocks(B.mx4_empty, ROWS, K), blocks(B.mx4_empty, N, K), blocks(B.ckpt8_empty, N, K))


def calls(x, y, kept, q, w, dx, dw, v):
    """Every call that takes blocks, by its name."""
    return {"aq_layernorm_forward": lambda: B.layernorm_forward(x, None, None, 1e-5, dx, v, v, kept),
            "aq_layernorm_backward": lambda: B.layernorm_backward(x, kept, None, v, v, dx, None, None),
            "aq_ckpt8_pack": lambda: B.ckpt8_pack(x, kept),
            "aq_ckpt8_unpack": lambda: B.ckpt8_unpack(kept, x),
            "aq_ckpt8_weight_grad": lambda: B.ckpt8_weight_grad(y, kept, dw),
            "aq_mx4_quantize": lambda: B.mx4_quantize(x, q),
            "aq_mx4_dequantize": lambda: B.mx4_dequantize(q, x),
            "aq_mx4_linear": lambda: B.mx4_linear(x, w, None, y),
            "aq_mx4_matmul": lambda: B.mx4_matmul(q, w, None, y),
            "aq_mx4_input_grad": lambda: B.mx4_input_grad(y, w, dx)}


def test_each_call_takes_its_own_kind_of_blocks(lib):
    """A checkpoint's block has 32 bytes of codes and a 4-bit tensor's 16: one taken for the other is written or read behind its end."""
    x, y, kept, q, w, w8 = operands()
    v, dx, dw = torch.zeros(ROWS), torch.zeros(ROWS, K), torch.zeros(N, K)
    for name, call in calls(x, y, kept, q, w, dx, dw, v).items():
        call()
        assert lib.calls.pop() == name and not lib.calls
    wrong = calls(x, y, q, kept, w8, dx, dw, v)
    wrong["the weights alone"] = lambda: B.mx4_matmul(q, w8, None, y)
    wrong["the input alone"] = lambda: B.mx4_matmul(kept, w, None, y)
    for name, call in wrong.items():
        with pytest.raises(ValueError, match="8-bit checkpoint|4-bit tensor"):
            call()
        assert not lib.calls, name
    for other in (None, x):  # no blocks at all
        for name, call in calls(x, y, other, other, other, dx, dw, v).items():
            if "layernorm" not in name:  # (forward keeps nothing then, backward reads a matrix)
                with pytest.raises(ValueError, match="8-bit checkpoint|4-bit tensor"):
                    call()
                assert not lib.calls, name
