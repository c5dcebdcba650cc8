"""Host code of the learner's operators on a HIP runtime of host memory (fake_hip.c): which kernels a call launches, on which tiles and in
how many slices.  Each scenario runs in a process of its own, in which no other HIP runtime is loaded."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
from test_host_routes import LAUNCH, Host, fake  # noqa: E402,F401

TYPES = {"f32": 0, "f16": 1, "bf16": 2}
A, SCALES, WS = 1 << 20, (1 << 20) + 1, 1 << 40  # addresses that nothing reads


class Learner(Host):
    def __init__(self, fake_path):
        super().__init__(fake_path)
        self.lib = self.aq.load()

    def matrix(self, rows, cols, kind, ld=None):
        return C.byref(self.aq.AqMatrix(A, rows, cols, cols if ld is None else ld, TYPES[kind]))

    def blocks(self, rows, cols):
        return C.byref(self.aq.AqBlocks(A, SCALES, rows, cols))

    def call(self, fn, *args):
        """(status, launches)"""
        self.hip.fake_clear()
        status = getattr(self.lib, fn)(*args, None)
        return status, self.logged(LAUNCH)

    def weight_grad(self, rows, n, k, kind):
        size = self.aq.ckpt8_weight_grad_workspace(rows, n, k)
        return self.call("aq_ckpt8_weight_grad", self.matrix(rows, n, kind), self.blocks(rows, k), self.matrix(n, k, "f32"), A, WS, size)

    def input_grad(self, rows, n, k, kind):
        size = self.aq.mx4_input_grad_workspace(rows, n, k)
        return self.call("aq_mx4_input_grad", self.matrix(rows, n, kind), self.blocks(n, k), self.matrix(rows, k, kind), WS, size)

    def linear(self, rows, n, k, kind):
        size = self.aq.mx4_linear_workspace(rows, n, k)
        return self.call("aq_mx4_linear", self.matrix(rows, k, kind), self.blocks(n, k), A, self.matrix(rows, n, kind), WS, size)

    def matmul(self, rows, n, k, kind):
        return self.call("aq_mx4_matmul", self.blocks(rows, k), self.blocks(n, k), A, self.matrix(rows, n, kind))


def products_of_many_rows_and_few_columns(h):
    """A result is refused by its 256 x 256 tiles alone (2^23 of them and more), before anything is launched."""
    for rows, n, k in ((1 << 30, 40, 64), ((1 << 31) - 256, 1, 1), ((1 << 31) - 256, 40, 70), ((1 << 31) - 256, 256, 256), ((1 << 30) - 256, 512, 512)):
        for kind in TYPES:
            for call in (h.input_grad, h.linear, h.matmul):
                status, launches = call(rows, n, k, kind)
                assert status == h.aq.OK and launches, (call.__name__, rows, n, k, kind, status)
                assert all(e.name for e in launches)
    for call in (h.input_grad, h.linear, h.matmul):
        for rows, n, k in (((1 << 31) - 255, 257, 257), (1 << 30, 513, 513)):
            status, launches = call(rows, n, k, "bf16")
            assert status == h.aq.ESHAPE and not launches, (call.__name__, rows, n, k, status)


SCENARIOS = [products_of_many_rows_and_few_columns]


@pytest.mark.parametrize("name", [s.__name__ for s in SCENARIOS])
def test_host(fake, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    {s.__name__: s for s in SCENARIOS}[sys.argv[2]](Learner(sys.argv[1]))
