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
import learner_shapes as shapes  # noqa: E402
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


def gradients_on_every_tile(h):
    """The sizes of the tests reach every tile, several groups of wavefronts and several slices, for every type."""
    for fn, listed in ((h.weight_grad, shapes.WEIGHT_GRAD), (h.input_grad, shapes.INPUT_GRAD)):
        reached = set()
        for sizes, *plans in listed:
            rows, n, k = sizes
            m, c = (n, k) if fn == h.weight_grad else (rows, k)
            for kind, want in zip(TYPES, plans):
                status, launches = fn(rows, n, k, kind)
                side, groups = map(int, re.search(rb"Li(\d+)ELi(\d+)EE+v", launches[0].name).groups())
                slices, rest = divmod(launches[0].grid[0], -(-m // side) * -(-c // side))
                assert status == h.aq.OK and b"6k_gradI" in launches[0].name and rest == 0
                assert len(launches) == (2 if slices > 1 else 1) and all(b"k_grad_join" in e.name for e in launches[1:])
                assert (side, groups, slices > 1) == want and (slices == 1 or slices > 2), (fn.__name__, sizes, kind, side, groups, slices)
                reached.add((kind, *want))
        assert reached == {(kind, *tile, split) for kind in TYPES for tile in ((64, 1), (64, 2), (128, 1), (256, 1)) for split in (False, True)}


def products_on_every_tile(h):
    for sizes, side in shapes.MX4:
        for kind in TYPES:
            status, launches = h.matmul(*sizes, kind)
            assert status == h.aq.OK and len(launches) == 1
            found = re.search(rb"k_mx4_tilesI.*?Li(\d+)E", launches[0].name)
            assert (int(found[1]) if found else 0) == side and (found or b"k_mx4_rows" in launches[0].name), (sizes, kind, launches[0].name)


SCENARIOS = [gradients_on_every_tile, products_on_every_tile, products_of_many_rows_and_few_columns]


@pytest.mark.parametrize("name", [s.__name__ for s in SCENARIOS])
def test_host(fake, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    {s.__name__: s for s in SCENARIOS}[sys.argv[2]](Learner(sys.argv[1]))
