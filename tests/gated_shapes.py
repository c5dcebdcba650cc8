"""Sizes at which gated layers and the recurrence are tested, and what they are to reach there: the tests that run them (test_gpu_gated.py,
test_gpu_recurrence.py) and those that look at the launches (test_memory_routes.py) read the same lists."""

# gated layers, rows, n, k: together every tile of every product, in one slice and in several, and both gradients in one launch
GATED = [(8, 8, 8), (5, 8, 11), (5, 396, 799), (5, 709, 2173), (325, 4099, 8), (29024, 206, 10), (70, 1733, 3042), (13474, 76, 70), (3125, 481, 75), (546, 225, 2950),
         (12422, 10, 2492), (442, 3504, 4404), (5579, 392, 2527)]

# the recurrence: sequences, their mean rows, units, whether they are ragged; then units of a lane, wavefronts forward and backward, and how
# sequences are taken ("each", "parts", "ordered")
RECURRENCE = [
    ((5, 1, 34, False), 1, 1, 1, "each"), ((5, 16, 34, False), 1, 1, 2, "each"), ((5, 31, 34, True), 1, 2, 4, "each"),
    ((5, 60, 34, False), 1, 4, 8, "each"), ((5, 130, 34, False), 1, 8, 8, "each"), ((5, 300, 34, False), 1, 8, 8, "parts"),
    ((5, 300, 35, True), 1, 4, 8, "parts"), ((1, 2100, 66, True), 1, 4, 8, "parts"),
    ((64, 1, 1024, False), 2, 1, 1, "each"), ((64, 9, 1025, False), 2, 2, 2, "each"), ((64, 30, 1024, False), 2, 4, 4, "each"),
    ((64, 70, 1026, False), 2, 8, 8, "each"), ((64, 66, 1023, True), 1, 8, 8, "ordered"), ((600, 5, 1000, True), 2, 1, 1, "each"),
    ((8, 1500, 1024, False), 2, 8, 8, "parts"), ((520, 64, 1024, True), 2, 4, 4, "ordered"),
    ((600, 30, 1000, True), 2, 2, 2, "each"), ((260, 100, 1024, True), 2, 4, 4, "ordered"), ((260, 128, 1024, True), 1, 8, 8, "ordered"),
]
