"""Products whose sizes reach each kernel and each way of cutting a product, and which one that is.

P columns and Q rows of the output, K long: a forward product has n = P, rows = Q, k = K, an input gradient
k = P, rows = Q, n = K, a weight gradient k = P, n = Q, rows = K.  "256/1" is the kernel of 256 x 256 tiles, its
reduction whole; "256/3": all of its tiles in 3 parts; "256+3": whole tiles, and a last round in 3 parts.  "128"
has two workgroups a CU, "deep" one; "any" operands of any alignment; "few1x16" rows straight from registers, 1 x 16
rows and 16 columns a workgroup."""

# P, Q, K, padding of a row, the first element's offset: 8-element vectors throughout
TILES_256 = [
    (2056, 4083, 392, 0, 0, "256/1"),         # 7 steps; one tile of 8 columns, one of 243 rows, a step of 8
    (2056, 4083, 456, 8, 8, "256/1"),         # 8 steps
    (2056, 1003, 14984, 0, 0, "256/7"),
    (4360, 4333, 4104, 8, 0, "256+4"),
    (5112, 14301, 1272, 0, 0, "256/1"),       # five rounds
    (1272, 14301, 5112, 0, 0, "256+8"),
]
# weight gradients: Q a multiple of 8, any K
WGRAD_256 = [
    (2056, 4088, 391, 0, 0, "256/1"),
    (2056, 4088, 453, 8, 8, "256/1"),
    (4360, 4360, 4099, 8, 0, "256+3"),
    (1272, 5112, 14301, 0, 0, "256/2"),
]
# (from here on a checkpoint's product is cut otherwise)
WGRAD_256_BF16 = [(2056, 1000, 14981, 0, 0, "256/7")]
WGRAD_256_CKPT = [(2056, 2000, 5121, 0, 0, "256/3"), (2056, 2056, 8205, 8, 8, "256/3")]
# smaller tiles: whole, in parts, and a last round in parts
TILES_128 = [(2056, 4090, 1416, 0, 0, "128+5"), (1288, 1537, 7368, 8, 0, "128/3"), (2568, 1537, 200, 0, 8, "128/1"),
             (2568, 1537, 2888, 0, 0, "deep+6"), (776, 515, 2440, 8, 8, "deep/4")]

# rows, n, k, padding
FEW = [
    (1, 5120, 1280, 0, "few1x16"), (16, 5120, 1280, 8, "few1x16"), (7, 4088, 264, 0, "few1x16"), (15, 4104, 72, 0, "few1x16"),
    (3, 51864, 64, 0, "few1x16"),
    (17, 384, 1280, 0, "few2x8"), (31, 384, 72, 8, "few2x8"), (32, 1280, 1280, 0, "few2x8"), (25, 136, 2568, 0, "few2x8"),
    (17, 5120, 1280, 0, "few2x16"), (32, 5120, 1280, 8, "few2x16"), (17, 4104, 1280, 0, "few2x16"), (32, 4104, 200, 0, "few2x16"),
    (1, 4080, 200, 0, "few1x8"), (16, 136, 2568, 8, "few1x8"),
    (33, 5120, 1280, 0, "deep/1"), (33, 384, 1280, 8, "deep/5"),
]

# rows, n, k, padding, offset: sizes and strides that allow no vectors, the reduction in parts
ANY_FWD = [(130, 129, 1001, 3, 1, "any/4"), (40, 200, 2049, 5, 0, "any/7"), (257, 72, 4099, 0, 3, "any/13")]
ANY_DGRAD = [(33, 1001, 77, 3, 0, "any/4"), (70, 2049, 203, 0, 1, "any/7"), (48, 51866, 136, 0, 0, "any/63"),
             (1499, 1283, 1001, 3, 0, "any/3")]
ANY_WGRAD = [(1500, 283, 201, 3, 1, "any/6"), (1499, 1283, 1001, 3, 0, "any/4"), (2049, 40, 131, 0, 0, "any/7"),
             (513, 131, 7, 1, 1, "any/2")]
# ... of a weight gradient from a checkpoint: dy alone has no vectors
ANY_WGRAD_CKPT = [(1500, 283, 201, 3, 1, "any/6"), (1499, 1283, 1001, 3, 0, "any/2"), (2049, 37, 136, 0, 0, "any/7"),
                  (513, 131, 8, 1, 1, "any/2")]

# reductions of 1 to 7 steps, and in parts of which the last has 1 to 5: P = 136, Q = 40
STEPS = [8, 72, 136, 200, 264, 328, 392, 904, 968, 1032, 1096, 1288]
