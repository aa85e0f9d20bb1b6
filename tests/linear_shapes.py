"""Shapes that the linear gradients' rule on sizes sends to the wide tile: (workers' rows, features, outputs), by dy's type.

Listed once for the test of the rule (on the CPU) and for the kernels' test.
"""

WIDE_ONE_PART = {
    "bf16": [([130] * 38 + [0, 260], 520, 260),          # whole tiles and edges, even
             ([1, 0, 63, 64, 65] + [200] * 37, 515, 259),  # odd in both, ragged rows
             ([150] * 42, 513, 257)],
    "f32": [([130] * 26 + [0, 260], 520, 260),
            ([1, 0, 63, 64, 65] + [200] * 23, 515, 259),
            ([150] * 28, 512, 257)],
}
WIDE_IN_PARTS = {
    "bf16": [([13001, 10999], 1540, 130), ([12033, 12000], 1531, 131)],
    "f32": [([2731, 2600, 2669], 777, 771), ([2667] * 3, 1030, 600)],
}
