"""Sizes at which the products of the learner's operators are tested, and the kernels that they are to reach there: the tests that run
them (test_gpu_learner_tiles.py) and those that look at the launches (test_learner_routes.py) read the same list."""

# ckpt8_weight_grad: (rows, n, k), then for f32, f16 and bf16 the side of the tile, the groups of wavefronts that share one and whether the
# rows are split into slices
WEIGHT_GRAD = [
    ((263, 33, 37), (64, 1, True), (64, 2, False), (64, 2, False)),
    ((235, 33, 49), (64, 2, False), (64, 2, False), (64, 2, False)),
    ((1007, 541, 75), (64, 2, True), (64, 2, True), (64, 1, True)),
    ((257, 5703, 165), (64, 1, False), (64, 1, False), (64, 1, False)),
    ((2861, 65, 2155), (128, 1, True), (64, 1, True), (128, 1, True)),
    ((203, 4431, 655), (128, 1, False), (128, 1, False), (128, 1, False)),
    ((201, 1517, 5457), (256, 1, False), (256, 1, False), (256, 1, False)),
    ((4727, 141, 2951), (256, 1, True), (256, 1, True), (256, 1, True)),
    ((5385, 1605, 83), (64, 2, True), (128, 1, True), (64, 2, True)),
]
# mx4_input_grad: (rows, n, k) and the same of the n (n a multiple of 8: rows end with a piece of eight values)
INPUT_GRAD = [
    ((71, 205, 37), (64, 2, False), (64, 2, False), (64, 2, False)),
    ((73, 525, 33), (64, 1, True), (64, 1, True), (64, 1, True)),
    ((577, 3439, 33), (64, 2, True), (64, 2, True), (64, 2, True)),
    ((9421, 317, 71), (64, 1, False), (64, 1, False), (64, 1, False)),
    ((12961, 203, 221), (128, 1, False), (128, 1, False), (128, 1, False)),
    ((12961, 208, 221), (128, 1, False), (128, 1, False), (128, 1, False)),
    ((1681, 5669, 77), (128, 1, True), (128, 1, True), (128, 1, True)),
    ((1681, 5672, 77), (128, 1, True), (128, 1, True), (128, 1, True)),
    ((9561, 215, 779), (256, 1, False), (256, 1, False), (256, 1, False)),
    ((9561, 216, 779), (256, 1, False), (256, 1, False), (256, 1, False)),
    ((131, 4797, 3305), (256, 1, True), (256, 1, True), (256, 1, True)),
    ((131, 4800, 3305), (256, 1, True), (256, 1, True), (256, 1, True)),
]
# mx4_linear and mx4_matmul: (rows, n, k), the side of mx4_matmul's tile (0: the kernel for few rows).  64: every number of blocks above 16,
# modulo 16; all: several chunks of 8 blocks, odd numbers of them too
MX4 = [((1009, 1111, 32 * b - b % 5), 64) for b in (1, 2, 3, 5, 6, 7, 8, 9, 11, 13, 14, 15, *range(16, 33), 41)] + [
    ((2051, 2100, 1100), 128), ((2053, 2111, 1339), 128), ((2051, 2100, 249), 128),
    ((4101, 4099, 1700), 256), ((4099, 4131, 530), 256), ((4101, 4099, 255), 256),
    ((17, 40, 2001), 0), ((131, 300, 777), 0),
]
