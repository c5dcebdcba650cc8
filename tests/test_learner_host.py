"""What the learner's operators refuse, and the sizes they ask for (no GPU work: refused calls return before any)."""
import ctypes as C

import pytest

from paper_1910_01055_amd import binding as B

M, K = B.AqMatrix, B.AqBlocks


def mat(rows, cols, dtype=0, ld=None, d=0x10000):
    return C.byref(M(d, rows, cols, cols if ld is None else ld, dtype))


def blk(rows, cols, codes=0x20000, scales=0x30001):
    return C.byref(K(codes, scales, rows, cols))


BAD_MATRICES = [(None, B.EINVAL), (mat(4, 32, d=None), B.EINVAL), (mat(-1, 32), B.EINVAL), (mat(4, -1), B.EINVAL), (mat(4, 32, ld=31), B.EINVAL),
                (mat(4, 32, dtype=3), B.EINVAL), (mat(4, 32, dtype=-1), B.EINVAL), (mat(4, 32, d=0x10002), B.EINVAL),
                (mat(4, 32, dtype=2, d=0x10001), B.EINVAL), (mat(4, 0), B.ESHAPE), (mat(4, (1 << 20) + 1), B.ESHAPE),
                (mat(1 << 31, 32), B.ESHAPE), (mat(4, 32, ld=(1 << 21) + 1), B.ESHAPE)]
BAD_BLOCKS = [(None, B.EINVAL), (blk(4, 32, codes=None), B.EINVAL), (blk(4, 32, scales=None), B.EINVAL), (blk(4, 32, codes=0x20008), B.EINVAL),
              (blk(-1, 32), B.EINVAL), (blk(4, -1), B.EINVAL), (blk(4, 0), B.ESHAPE), (blk(4, (1 << 20) + 1), B.ESHAPE), (blk(1 << 31, 32), B.ESHAPE)]
V = 0x40000  # a vector
WS = 0x50000


@pytest.fixture(scope="module")
def lib():
    return B.load()


def test_matrices_and_blocks(lib):
    for m, want in BAD_MATRICES:
        assert lib.aq_ckpt8_pack(m, blk(4, 32), None) == want
        assert lib.aq_mx4_dequantize(blk(4, 32), m, None) == want
        assert lib.aq_layernorm_forward(m, V, V, 1e-5, mat(4, 32), V, V, None, None) == want
        assert lib.aq_layernorm_forward(mat(4, 32), V, V, 1e-5, m, V, V, None, None) == want
        assert lib.aq_layernorm_backward(m, mat(4, 32), None, V, V, V, mat(4, 32), V, V, WS, 1 << 30, None) == want
        assert lib.aq_layernorm_backward(mat(4, 32), mat(4, 32), None, V, V, V, m, V, V, WS, 1 << 30, None) == want
        assert lib.aq_ckpt8_weight_grad(m, blk(4, 32), mat(32, 32), V, WS, 1 << 30, None) == want
        assert lib.aq_ckpt8_weight_grad(mat(4, 32), blk(4, 32), m, V, WS, 1 << 30, None) == want
        assert lib.aq_mx4_linear(m, blk(32, 32), V, mat(4, 32), WS, 1 << 30, None) == want
        assert lib.aq_mx4_linear(mat(4, 32), blk(32, 32), V, m, WS, 1 << 30, None) == want
        assert lib.aq_mx4_matmul(blk(4, 32), blk(32, 32), V, m, None) == want
        assert lib.aq_mx4_input_grad(m, blk(32, 32), mat(4, 32), WS, 1 << 30, None) == want
        assert lib.aq_mx4_input_grad(mat(4, 32), blk(32, 32), m, WS, 1 << 30, None) == want
    for b, want in BAD_BLOCKS:
        assert lib.aq_ckpt8_pack(mat(4, 32), b, None) == want
        assert lib.aq_ckpt8_unpack(b, mat(4, 32), None) == want
        assert lib.aq_mx4_quantize(mat(4, 32), b, None) == want
        assert lib.aq_ckpt8_weight_grad(mat(4, 32), b, mat(32, 32), V, WS, 1 << 30, None) == want
        assert lib.aq_mx4_linear(mat(4, 32), b, V, mat(4, 32), WS, 1 << 30, None) == want
        assert lib.aq_mx4_matmul(b, blk(32, 32), V, mat(4, 32), None) == want
        assert lib.aq_mx4_input_grad(mat(4, 32), b, mat(4, 32), WS, 1 << 30, None) == want
        if b is not None:
            assert lib.aq_layernorm_forward(mat(4, 32), V, V, 1e-5, mat(4, 32), V, V, b, None) == want
            assert lib.aq_layernorm_backward(mat(4, 32), None, b, V, V, V, mat(4, 32), V, V, WS, 1 << 30, None) == want


def test_operands_that_do_not_go_together(lib):
    E = B.ESHAPE
    for other in (mat(5, 32), mat(4, 31), mat(4, 32, dtype=1)):
        assert lib.aq_layernorm_forward(mat(4, 32), V, V, 1e-5, other, V, V, None, None) == E
        assert lib.aq_layernorm_backward(mat(4, 32), other, None, V, V, V, mat(4, 32), V, V, WS, 1 << 30, None) == E
        assert lib.aq_layernorm_backward(mat(4, 32), mat(4, 32), None, V, V, V, other, V, V, WS, 1 << 30, None) == E
        assert lib.aq_mx4_linear(mat(4, 40), blk(32, 40), V, other, WS, 1 << 30, None) == E
        assert lib.aq_mx4_input_grad(mat(4, 40), blk(40, 32), other, WS, 1 << 30, None) == E
    for other in (blk(5, 32), blk(4, 31)):
        assert lib.aq_ckpt8_pack(mat(4, 32), other, None) == E
        assert lib.aq_ckpt8_unpack(other, mat(4, 32), None) == E
        assert lib.aq_mx4_quantize(mat(4, 32), other, None) == E
        assert lib.aq_mx4_dequantize(other, mat(4, 32), None) == E
        assert lib.aq_layernorm_forward(mat(4, 32), V, V, 1e-5, mat(4, 32), V, V, other, None) == E
        assert lib.aq_layernorm_backward(mat(4, 32), None, other, V, V, V, mat(4, 32), V, V, WS, 1 << 30, None) == E
    assert lib.aq_ckpt8_weight_grad(mat(4, 21), blk(5, 32), mat(21, 32), V, WS, 1 << 30, None) == E
    assert lib.aq_ckpt8_weight_grad(mat(4, 21), blk(4, 32), mat(20, 32), V, WS, 1 << 30, None) == E
    assert lib.aq_ckpt8_weight_grad(mat(4, 21), blk(4, 32), mat(21, 33), V, WS, 1 << 30, None) == E
    assert lib.aq_ckpt8_weight_grad(mat(4, 21), blk(4, 32), mat(21, 32, dtype=2), V, WS, 1 << 30, None) == E
    assert lib.aq_mx4_linear(mat(4, 33), blk(21, 32), V, mat(4, 21), WS, 1 << 30, None) == E
    assert lib.aq_mx4_matmul(blk(4, 33), blk(21, 32), V, mat(4, 21), None) == E
    assert lib.aq_mx4_matmul(blk(4, 32), blk(21, 32), V, mat(4, 20), None) == E
    assert lib.aq_mx4_input_grad(mat(4, 20), blk(21, 32), mat(4, 32), WS, 1 << 30, None) == E
    wide = (1 << 14) + 1
    assert lib.aq_layernorm_forward(mat(4, wide), V, V, 1e-5, mat(4, wide), V, V, None, None) == E
    assert lib.aq_layernorm_backward(mat(4, wide), mat(4, wide), None, V, V, V, mat(4, wide), V, V, WS, 1 << 30, None) == E


def test_vectors_scratch_and_the_rest(lib):
    E = B.EINVAL
    m = mat(4, 32)
    for i in range(4):
        v = [V + (2 if j == i else 0) for j in range(4)]
        assert lib.aq_layernorm_forward(m, v[0], v[1], 1e-5, m, v[2], v[3], None, None) == E
    for eps in (-1e-5, float("nan")):
        assert lib.aq_layernorm_forward(m, V, V, eps, m, V, V, None, None) == E
    for i in range(5):
        v = [V + (2 if j == i else 0) for j in range(5)]
        assert lib.aq_layernorm_backward(m, m, None, v[0], v[1], v[2], m, v[3], v[4], WS, 1 << 30, None) == E
    assert lib.aq_layernorm_backward(m, m, blk(4, 32), V, V, V, m, V, V, WS, 1 << 30, None) == E  # both
    assert lib.aq_layernorm_backward(m, None, None, V, V, V, m, V, V, WS, 1 << 30, None) == E  # neither
    assert lib.aq_layernorm_backward(m, m, None, V, None, V, m, V, V, WS, 1 << 30, None) == E
    assert lib.aq_layernorm_backward(m, m, None, V, V, None, m, V, V, WS, 1 << 30, None) == E
    assert lib.aq_ckpt8_weight_grad(m, blk(4, 32), mat(32, 32), V + 1, WS, 1 << 30, None) == E
    assert lib.aq_mx4_linear(m, blk(32, 32), V + 2, m, WS, 1 << 30, None) == E
    assert lib.aq_mx4_matmul(blk(4, 32), blk(32, 32), V + 2, m, None) == E
    # scratch: too little, none, or one that starts anywhere
    big, y = mat(4096, 512), mat(4096, 512)
    sizes = (B.layernorm_backward_workspace(4096, 512), B.ckpt8_weight_grad_workspace(4096, 512, 512), B.mx4_linear_workspace(4096, 512, 512))
    assert all(s > 0 for s in sizes)
    calls = (lambda p, s: lib.aq_layernorm_backward(big, big, None, V, V, V, y, V, V, p, s, None),
             lambda p, s: lib.aq_ckpt8_weight_grad(big, blk(4096, 512), mat(512, 512), V, p, s, None),
             lambda p, s: lib.aq_mx4_linear(big, blk(512, 512), V, y, p, s, None))
    for call, size in zip(calls, sizes):
        assert call(WS, size - 1) == E and call(None, size) == E and call(WS + 8, size) == E and call(WS, 0) == E
    n = C.c_uint64(0)
    for fn, head in (("aq_layernorm_backward_workspace", ()), ("aq_ckpt8_weight_grad_workspace", (7,)), ("aq_mx4_linear_workspace", (7,)),
                     ("aq_mx4_input_grad_workspace", (7,))):
        f = getattr(lib, fn)
        assert f(5, *head, 9, C.byref(n)) == B.OK and f(0, *head, 9, C.byref(n)) == B.OK
        assert f(5, *head, 9, None) == E and f(-1, *head, 9, C.byref(n)) == E and f(5, *head, -9, C.byref(n)) == E
        assert f(5, *head, 0, C.byref(n)) == B.ESHAPE and f(1 << 31, *head, 9, C.byref(n)) == B.ESHAPE
        assert f(5, *head, (1 << 20) + 1, C.byref(n)) == B.ESHAPE


def test_no_gpu_is_an_error_not_a_fallback(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("has a GPU")
    assert lib.aq_mx4_matmul(blk(4, 32), blk(32, 32), None, mat(4, 32), None) == B.EHIP
    assert lib.aq_layernorm_forward(mat(4, 32), None, None, 1e-5, mat(4, 32), None, None, None, None) == B.EHIP


def test_the_binding_checks_tensors():
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        B._matrix(x.t())  # columns, not rows, are contiguous
    with pytest.raises(ValueError):
        B._matrix(x.double())
    with pytest.raises(ValueError):
        B._matrix(x[0])
    m = M.from_buffer_copy(B._matrix(x[:, 3:40]))
    assert (m.rows, m.cols, m.ld, m.dtype) == (4, 37, 64, 0) and m.d == x.data_ptr() + 12
    with pytest.raises(ValueError):
        B._vector(torch.zeros(5), 4, "v")
    with pytest.raises(ValueError):
        B._vector(torch.zeros(8)[::2], 4, "v")
    with pytest.raises(ValueError):
        B._vector(torch.zeros(4, dtype=torch.float16), 4, "v")
    for make in (B.ckpt8_empty, B.mx4_empty):
        q = make(3, 70, device="cpu")
        c = K.from_buffer_copy(q._c)
        assert (c.rows, c.cols) == (3, 70) and c.d_codes == q.codes.data_ptr() and c.d_scales == q.scales.data_ptr()
        assert tuple(q.scales.shape) == (3, 3) and q.codes.shape[1] == 3 * q.CODE_BYTES
        with pytest.raises(ValueError):
            type(q)(q.codes, q.scales, 97)
        with pytest.raises(ValueError):
            type(q)(q.codes[:, 1:], q.scales, 70)
