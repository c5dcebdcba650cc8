"""Host code of the gated layers and the recurrence on a HIP runtime of host memory (fake_hip.c): which kernels a call launches.  Each
scenario runs in a process of its own, in which no other HIP runtime is loaded."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
import gated_shapes as shapes  # noqa: E402
from test_host_routes import fake  # noqa: E402,F401
from test_learner_routes import TYPES, WS, A, Learner  # noqa: E402


class Memory(Learner):
    def names(self, fn, *args):
        status, launches = self.call(fn, *args)
        return status, [bytes(e.name) for e in launches], [e.grid[0] for e in launches]

    def gated(self, rows, n, k, kind):
        """The launches of both passes."""
        M, size = self.matrix, C.c_uint64()
        assert self.lib.aq_gated_forward_workspace(rows, n, k, TYPES[kind], C.byref(size)) == 0
        m, w, x = M(rows, n, kind), M(n, k, kind), M(rows, k, kind)
        forward = self.names("aq_gated_forward", x, w, w, 1, m, m, m, WS, size.value)
        assert self.lib.aq_gated_backward_workspace(rows, n, k, TYPES[kind], C.byref(size)) == 0
        backward = self.names("aq_gated_backward", m, x, w, w, m, m, 1, x, w, w, WS, size.value)
        return forward, backward

    def recurrence(self, count, mean, c, ragged, kind, starts=None):
        M, size, rows = self.matrix, C.c_uint64(), count * mean
        assert self.lib.aq_recurrence_workspace(rows, count, c, C.byref(size)) == 0
        m, off = M(rows, c, kind), A if ragged else None
        forward = self.names("aq_recurrence_forward", m, m, off, count, starts, 1 << 20, m, 2 << 20, WS, size.value)
        backward = self.names("aq_recurrence_backward", m, None, m, m, m, off, count, starts, None, m, m, None, WS, size.value)
        return forward, backward


PRODUCT = re.compile(rb"k_gated_productI.*?Li(\d+)ELNS_4FormE(\d)ELb(\d)E")
GRADIENTS = re.compile(rb"k_gated_gradientsI.*?Li(\d+)ELi\dE")


def reached_by(kind, sizes, launches):
    """The products of a call's launches: type, tile, form (0 forward, 1 input, 2 weights, 3 both gradients in one launch), then what is joined:
    0 nothing, 1 the product (the input's gradient), 2 the weights' gradients, 3 all."""
    rows, n, k = sizes
    _, names, grids = launches
    for i, name in enumerate(names):
        follows = names[i + 1] if i + 1 < len(names) else b""
        found, pair = PRODUCT.search(name), GRADIENTS.search(name)
        if found:
            assert (b"k_gated_join" in follows) == (found[3] == b"1"), names
            yield (kind, *map(int, found.groups()))
        elif pair:
            size, blocks = int(pair[1]), lambda v: -(-v // 256)
            joins = {0: 0, blocks(rows * k): 1, blocks(2 * n * k): 2, blocks(rows * k + 2 * n * k): 3}
            alone = [b"k_gated_gradients" in m or b"k_gated_productI" in m for m in names].count(True) > 1
            form = 3 if not alone else 1 if b"slopes" in names[i - 1] else 2
            joined = joins[grids[i + 1]] if b"k_gated_join" in follows else 0
            yield (kind, size, form, joined)


def gated_products(h):
    """The sizes of the tests reach every tile of every product, in one slice and in several, for every type, alone and with both gradients
    in one launch; few rows have a kernel of their own, and rows that are no whole pieces are laid out first."""
    reached = set()
    for sizes in shapes.GATED:
        for kind in TYPES:
            for launches in h.gated(*sizes, kind):
                assert launches[0] == h.aq.OK
                reached |= set(reached_by(kind, sizes, launches))
    wanted = {(k, s, 0, p) for k in TYPES for s in ((64, 128) if k == "f32" else (64, 128, 256)) for p in (0, 1)}
    wanted |= {(k, 256, f, p) for k in ("f16", "bf16") for f in (1, 2) for p in (0, 1)}
    wanted |= {(k, s, 3, p) for k in TYPES for s in (64, 128) for p in (0, 1, 2, 3)}
    assert wanted <= reached, sorted(wanted - reached)
    for kind in TYPES:
        for rows in (1, 2, 3, 4):
            _, names, _ = h.gated(rows, 40, 77, kind)[0]
            assert len(names) == 1 and b"k_gated_rows" in names[0]
        _, names, _ = h.gated(40, 40, 80, kind)[0]
        assert any(b"k_lay_out" in n for n in names) == (kind == "f32")
        _, names, _ = h.gated(40, 40, 81, kind)[0]
        assert any(b"k_lay_out" in n for n in names)


def gated_sizes(h):
    """As many rows and features as a launch holds, and none."""
    for rows, n, k in (((1 << 31) - (1 << 20), 1, 4), (1 << 27, 64, 8), (5, 1 << 20, 1), (1, 1 << 20, 8192), (0, 5, 7), (100, 8192, 1 << 20)):
        for kind in TYPES:
            for status, names, _ in h.gated(rows, n, k, kind):
                assert status == h.aq.OK and bool(names) == (rows > 0 or b"k_gated_gradients" in b"".join(names)), (rows, n, k, kind, status)
    size = C.c_uint64()
    for rows, n, k in ((1 << 27, 65, 8), (1 << 27, 8, 65), (8, 1 << 20, 8193)):
        assert h.lib.aq_gated_forward_workspace(rows, n, k, 2, C.byref(size)) == h.aq.ESHAPE
        assert h.lib.aq_gated_backward_workspace(rows, n, k, 2, C.byref(size)) == h.aq.ESHAPE


def recurrences(h):
    for (count, mean, c, ragged), units, forward, backward, how in shapes.RECURRENCE:
        for kind in TYPES:
            for starts in (None, A):
                for (status, names, grids), waves, fn in zip(h.recurrence(count, mean, c, ragged, kind, starts), (forward, backward), (b"k_recurrenceI", b"k_recurrence_backwardI")):
                    where = (count, mean, c, ragged, kind, fn, names)
                    assert status == h.aq.OK, where
                    sums = names[0] if how == "parts" else None
                    assert len(names) == (1 if how == "each" else 2) and (how != "ordered" or b"k_recurrence_order" in names[0]), where
                    found = re.search(rb"Li(\d)ELi\d+ELi(\d)ELb(\d)ELb(\d)E", names[-1])
                    assert fn in names[-1] and tuple(map(int, found.groups())) == (units, waves, 0, starts is not None), where
                    assert sums is None or (fn in sums and re.search(rb"ELb(\d)ELb\dE", sums)[1] == b"1"), where
                    lanes = (c + units - 1) // units
                    assert how == "parts" or grids[-1] == -(-count * lanes // 64), where


SCENARIOS = [gated_products, gated_sizes, recurrences]


@pytest.mark.parametrize("name", [s.__name__ for s in SCENARIOS])
def test_host(fake, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, name], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    {s.__name__: s for s in SCENARIOS}[sys.argv[2]](Memory(sys.argv[1]))
