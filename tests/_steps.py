"""Sizes of steps that reach every tile of the products, split and not, in one tile a
workgroup and in several (test_plan checks that they do)."""

LAYER_STEPS = [
    # M, K, N, dy, dx
    (131, 1455, 1429, "f32", "f32"), (277, 3497, 1165, "f32", "f32"),
    (261, 1033, 7327, "bf16", "bf16"), (31117, 827, 145, "f32", "f32"),
    (65, 4983, 5549, "bf16", "f32"), (39835, 769, 135, "bf16", "bf16"),
    (16685, 4809, 69, "f32", "bf16"), (1325, 867, 5623, "f32", "bf16"),
    (38931, 797, 257, "bf16", "f32"), (4099, 2305, 511, "bf16", "bf16"),
]
LOSS_STEPS = [
    # M, K, V, x, w, dx, dw
    (75, 201, 151, "f32", "f32", "bf16", "f32"), (253, 591, 141, "bf16", "bf16", "f32", "bf16"),
    (17947, 203, 75, "bf16", "f32", "f32", "f32"), (5711, 531, 129, "f32", "f32", "f32", "f32"),
    (34495, 215, 77, "f32", "f32", "f32", "f32"), (993, 203, 8467, "f32", "f32", "f32", "f32"),
    (1087, 251, 6769, "f32", "bf16", "bf16", "f32"), (33107, 477, 287, "f32", "f32", "f32", "f32"),
    (321, 5417, 1341, "f32", "f32", "f32", "bf16"), (149, 3307, 5689, "f32", "f32", "f32", "bf16"),
    (1293, 5887, 93, "f32", "f32", "f32", "f32"), (69, 4807, 6143, "f32", "f32", "f32", "f32"),
    (4665, 201, 5229, "f32", "f32", "bf16", "bf16"),
    # operands that are read as they lie
    (2047, 576, 6001, "bf16", "bf16", "bf16", "bf16"),
]
# More than one piece of the classes: of many rows two and three, of few rows pieces so long
# that dx is split, its sums over the earlier pieces added where the splits are joined
PIECES = [
    # M, K, V, x, w, dx, dw, pieces
    (20000, 9, 4500, "f32", "f32", "f32", "f32", 2),
    (45001, 24, 4301, "f32", "bf16", "f32", "f32", 3),
    (66001, 128, 4517, "bf16", "bf16", "bf16", "bf16", 3),
    (33000, 70, 4200, "bf16", "f32", "bf16", "bf16", 2),
    (3, 16, 1400003, "f32", "f32", "f32", "f32", 2),
    (70, 40, 2100001, "bf16", "bf16", "bf16", "bf16", 3),
]
