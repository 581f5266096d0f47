"""Sizes of the operators' matrix products and the tiles that they take on 256 compute
units (csrc_ops/mm_shape.h), none a whole number of tiles: test_operators_tiles_cpu
holds the rule to this table, test_gpu_operators_tiles runs the sizes."""

UNITS = 256

# (matrices, rows, columns): tiles of X X^T, of B = b A + c A^2 and of a X + B X (and the
# last step's, which writes the result)
ORTH = {
    (1, 67, 69): ("32 by 4", "32 by 4", "32 by 4"),
    (43, 65, 67): ("64 by 2", "64 by 2", "64 by 2"),
    (44, 129, 131): ("64", "64", "64"),
    (52, 131, 265): ("64", "64", "128"),
    (52, 129, 517): ("64", "64", "192"),
    (52, 258, 263): ("128", "128", "128"),
    (35, 513, 517): ("192", "192", "128"),
    (41, 515, 518): ("192", "192", "192"),
    (20, 770, 903): ("256", "256", "192"),
    (26, 707, 711): ("256", "256", "256"),
    (1, 1500, 3001): ("64", "64", "128"),
}
# ... of updates: each of the tiles that a last step may have
MUON = [(1, 67, 69), (43, 65, 67), (44, 129, 131), (52, 258, 263), (41, 515, 518), (26, 707, 711)]

# (rows, inputs, outputs)
LINEAR = {
    (18, 249, 25): "32 by 4",
    (33, 66, 4117): "64 by 2",
    (8219, 14, 70): "64",
    (7014, 14, 387): "128",
    (8221, 70, 977): "128 x 192",
    (10000, 500, 1021): "128 x 192",
    (8304, 30, 901): "192",
    (8286, 1411, 967): "256",
}
