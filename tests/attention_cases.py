"""Shapes (sequences, rows, keys, heads, key heads, d, dv) that reach each variant of differential attention on a device of 256
compute units; test_attention_variants checks that they do, test_gpu_attention_variants what the variants compute."""

# many rows a workgroup, in the width classes (32, 64) and (64, 128): tiles' ends, odd widths, shared keys, few keys
MANY_ROWS = [(64, 100, 100, 3, 3, 32, 64), (16, 130, 257, 6, 6, 32, 64), (48, 60, 90, 8, 4, 32, 64), (64, 70, 200, 3, 3, 20, 36),
             (64, 128, 64, 3, 3, 17, 33), (96, 65, 1, 2, 2, 8, 8),
             (8, 513, 513, 3, 3, 64, 128), (8, 200, 300, 8, 2, 64, 128), (24, 100, 140, 4, 4, 61, 107), (12, 129, 70, 4, 4, 40, 72),
             (32, 65, 33, 3, 3, 64, 128), (4, 1000, 77, 3, 3, 63, 127)]
# and in those of wider keys
MANY_ROWS_WIDE = [(64, 65, 70, 2, 2, 128, 128), (32, 70, 90, 4, 4, 100, 90), (32, 129, 64, 3, 3, 128, 256), (40, 100, 60, 4, 4, 97, 201)]
# many rows of sequences of unequal length: (shape, its rows and keys the longest)
PADDED = [(26, 150, 150, 4, 2, 64, 128), (33, 140, 140, 6, 3, 32, 64), (26, 135, 135, 2, 2, 61, 107), (33, 131, 131, 3, 3, 20, 36)]
PACKED = [(40, 300, 300, 4, 2, 64, 128), (40, 300, 300, 6, 6, 32, 64), (40, 300, 300, 4, 4, 61, 107), (40, 300, 300, 6, 6, 20, 36)]
# a key head that very many heads share, and one as a step of training has it
SHARED = [(1, 3, 70, 200, 1, 32, 64), (2, 40, 50, 70, 1, 64, 128), (1, 2, 40, 130, 2, 128, 200)]
STEP = (16, 150, 150, 6, 3, 64, 128)
# the keys of few rows in parts: (shape, whether lengths are given, parts)
PARTS = [((1, 1, 40000, 1, 1, 128, 256), False, 256), ((1, 1, 60000, 1, 1, 64, 128), False, 117), ((1, 1, 50000, 1, 1, 32, 64), False, 97),
         ((1, 2, 33000, 1, 1, 128, 128), False, 256), ((1, 40, 30000, 2, 1, 61, 107), False, 58),
         ((16, 1, 16384, 16, 4, 64, 128), True, 8), ((4, 1, 16500, 2, 2, 32, 64), True, 32), ((2, 3, 9000, 4, 2, 128, 256), True, 70)]
# the rows of few keys in parts: (shape, parts)
ROW_PARTS = [((1, 9000, 100, 1, 1, 64, 128), 64), ((1, 5000, 130, 2, 1, 32, 64), 64), ((1, 3000, 100, 1, 1, 128, 256), 23),
             ((2, 700, 300, 2, 2, 128, 128), 5), ((1, 4100, 70, 1, 1, 33, 65), 32)]
