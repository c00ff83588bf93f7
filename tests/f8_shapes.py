"""Calls of 8-bit products that take each kernel and tile: (rows, tiles of features, parts of the columns, row blocks) of f8_shape() in csrc/dispatch_rules.h -> samples, rows a sample, experts,
n, k, gated, products in fp32 sums."""
SHAPES = [
    # 128 x 256
    ((128, 16, 1, 0), (1290, 1, 1, 4100, 300, False, False)), ((128, 16, 1, 0), (1290, 1, 1, 2050, 300, True, False)), ((128, 16, 1, 0), (60, 31, 3, 2800, 130, False, False)),
    # 64 x 256
    ((64, 16, 1, 0), (150, 1, 1, 16001, 400, False, False)), ((64, 16, 1, 0), (150, 1, 1, 8010, 400, True, False)), ((64, 16, 1, 0), (1000, 1, 1, 6500, 640, False, True)),
    ((64, 16, 1, 0), (1000, 1, 1, 3250, 640, True, True)),
    # 64 x 128
    ((64, 8, 1, 0), (300, 1, 1, 4100, 1300, False, False)), ((64, 8, 1, 0), (300, 1, 1, 2050, 1300, True, False)), ((64, 8, 1, 0), (300, 1, 1, 4100, 513, False, True)),
    ((64, 8, 1, 0), (300, 1, 1, 2050, 513, True, True)),
    # 32 x 128, and its columns in two parts
    ((32, 8, 1, 0), (20, 1, 1, 20500, 700, False, False)), ((32, 8, 1, 0), (60, 1, 4, 5200, 700, False, True)), ((32, 8, 1, 0), (20, 1, 1, 10300, 700, True, False)), ((32, 8, 1, 0), (60, 1, 4, 2600, 700, True, True)),
    ((32, 8, 2, 0), (70, 1, 1, 900, 2000, True, False)), ((32, 8, 2, 0), (70, 1, 1, 900, 2000, True, True)),
    # 64 x 64 in two parts, 32 x 64 in four
    ((64, 4, 2, 0), (250, 1, 1, 3000, 1500, False, False)), ((64, 4, 2, 0), (250, 1, 1, 3000, 1500, False, True)),
    ((32, 4, 4, 0), (90, 1, 1, 1000, 2300, False, False)), ((32, 4, 4, 0), (90, 1, 1, 1000, 2300, False, True)),
    # few rows
    ((0, 1, 1, 1), (1, 1, 1, 3000, 2000, False, True)), ((0, 1, 1, 1), (12, 1, 1, 3000, 2000, False, False)), ((0, 2, 1, 1), (7, 1, 1, 9000, 900, False, True)), ((0, 2, 1, 1), (5, 1, 3, 1000, 900, True, False)),
    ((0, 2, 1, 1), (30, 1, 1, 700, 1700, False, False)), ((0, 2, 1, 1), (8, 1, 2, 1000, 900, True, True)), ((0, 2, 1, 2), (50, 1, 1, 700, 1700, False, False)), ((0, 2, 1, 2), (50, 1, 1, 700, 1700, False, True)),
]
