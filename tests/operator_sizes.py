"""Sizes by which the tests on the GPU reach the forms of the operators' kernels that only larger calls take, each with the form it is there for.
test_operator_launches.py holds the library to these."""

# n, dim, hidden, dtype, act, pad: what the products of the forward pass are (tiles of 256 or 128, and whether the tiles of a last, partly
# filled round are split over the inner dimension: all of them, those beyond whole rounds, or none)
FORWARD = {
    (7406, 1056, 1136, "bf16", "silu", 0): "256 rest split",
    (1500, 2048, 4096, "f16", "silu", 8): "256 unsplit",
    (137, 2542, 4432, "f16", "gelu", 3): "256 all split",
    (908, 95, 4239, "bf16", "gelu", 1): "256 unsplit",
    (3389, 3552, 1159, "bf16", "silu", 0): "128 rest split",
    (138, 1056, 116, "f16", "silu", 0): "128 all split",
    (163, 96, 108, "bf16", "gelu", 5): "128 unsplit",
}
# ... and of dx, and of dWg and dWu, each in a launch of its own
BACKWARD = {
    (1500, 2048, 4096, "bf16", "silu", 0): ("256 all split", "256 unsplit"),
    (1999, 1601, 4099, "f16", "gelu", 3): ("256 all split", "256 unsplit"),
    (1485, 1200, 6591, "bf16", "gelu", 8): ("256 all split", "256 rest split"),
    (9387, 1552, 940, "f16", "silu", 0): ("256 rest split", "256 all split"),
    (7300, 1776, 143, "bf16", "silu", 0): ("256 unsplit", "128 all split"),
    (4878, 2791, 145, "bf16", "gelu", 1): ("256 unsplit", "256 all split"),
    (3943, 670, 5651, "f16", "silu", 0): ("256 all split", "128 rest split"),
    (1355, 1104, 3472, "bf16", "silu", 0): ("128 all split", "128 unsplit"),
    (6257, 144, 4773, "bf16", "silu", 8): ("128 all split", "256 all split"),
    (9340, 767, 647, "f16", "gelu", 0): ("128 unsplit", "128 all split"),
    (5560, 1464, 2130, "bf16", "gelu", 0): ("128 rest split", "256 all split"),
}
# n, dim, hidden, dtype, act, pad of passes of few tokens backward: blocks of columns, and hidden elements of a share
FEW_BACKWARD = {
    (1, 4096, 11008, "bf16", "silu", 0): (8, 86),
    (1, 9, 17000, "f16", "gelu", 1): (1, 67),
    (3, 513, 1000, "f16", "silu", 0): (2, 4),
    (4, 1601, 17000, "bf16", "gelu", 3): (4, 67),
    (8, 4099, 2500, "bf16", "silu", 0): (9, 23),
    (8, 2056, 3333, "f16", "silu", 8): (5, 17),
    (9, 512, 17024, "bf16", "gelu", 0): (2, 67),
    (12, 4100, 5000, "f16", "gelu", 5): (17, 84),
    (16, 1601, 8199, "bf16", "silu", 0): (7, 57),
    (16, 257, 17000, "f16", "silu", 1): (2, 67),
}
# dtype, grad dtype, n, rows of the table, dim of table gradients: 16-byte pieces of a row that a lane of the sums takes
TABLE_GRADIENT = {
    ("bf16", "bf16", 6500, 57, 520): 2,
    ("bf16", "bf16", 7000, 900, 1023): 2,
    ("bf16", "bf16", 7001, 57, 1030): 4,
    ("bf16", "bf16", 3100, 900, 2056): 4,
    ("bf16", "bf16", 2100, 40, 4099): 4,
    ("f16", "f16", 9000, 2000, 1024): 2,
    ("f16", "f16", 6200, 900, 1531): 4,
    ("bf16", "f32", 6700, 57, 301): 2,
    ("bf16", "f32", 7000, 900, 1030): 4,
    ("f16", "f32", 6500, 900, 512): 2,
    ("f16", "f32", 8191, 3000, 768): 4,
    ("f16", "f32", 2500, 40, 2051): 4,
    ("f32", "f32", 6500, 57, 260): 2,
    ("f32", "f32", 9000, 900, 511): 2,
    ("f32", "f32", 6600, 57, 515): 4,
    ("f32", "f32", 3300, 900, 1029): 4,
}
