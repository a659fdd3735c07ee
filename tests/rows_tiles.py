"""Sizes of the products whose rows choose their weights, and the tile that each runs on
256 compute units: tests/test_rows_plan.py holds the second to be true, and
tests/test_gpu_rows_tiles.py runs the first."""

# rows, n, k, groups: tile rows x columns, through registers, k slices. Rows of k and n
# bytes, dense; the groups' rows are uneven (test_gpu_rows_tiles.uneven).
GROUPED = {
    (1280, 1020, 260, 64): (32, 256, False, 1),
    (1281, 1021, 131, 64): (32, 256, True, 1),
    (900, 256, 384, 8): (64, 128, False, 1),
    (1000, 2100, 196, 20): (64, 128, False, 1),
    (1000, 2101, 129, 20): (64, 128, True, 1),
    (200, 130, 1030, 4): (64, 128, True, 3),
    (200, 132, 1028, 4): (64, 128, False, 3),
    (1300, 2300, 260, 5): (128, 128, False, 1),
    (4000, 1100, 132, 3): (128, 128, False, 1),
    (1300, 2301, 255, 5): (128, 128, True, 1),
    (4000, 3001, 97, 7): (128, 128, True, 1),
    (4000, 3000, 196, 7): (256, 256, False, 1),
    (5000, 2556, 128, 6): (256, 256, False, 1),
}

# m, n, k, adapters, rank: tile, through registers, k slices, u a row a workgroup, ranks a
# workgroup of u's blocks.
ADAPTERS = {
    (20, 65528, 36, 5, 8): (32, 256, False, 1, True, 16),
    (20, 65528, 36, 5, 250): (32, 256, False, 1, False, 16),
    (19, 65531, 33, 5, 7): (32, 256, True, 1, True, 16),
    (60, 65532, 40, 5, 8): (64, 128, False, 1, True, 16),
    (60, 65533, 37, 5, 8): (64, 128, True, 1, True, 16),
    (2000, 1020, 260, 30, 14): (64, 128, False, 1, False, 16),
    (2050, 2044, 132, 30, 8): (128, 128, False, 1, False, 16),
    (2050, 2044, 132, 30, 72): (128, 128, False, 1, False, 16),
    (2050, 2047, 65, 30, 21): (128, 128, True, 1, False, 16),
    (4000, 4092, 132, 40, 14): (256, 256, False, 1, False, 16),
    (4096, 4096, 1028, 3, 16): (256, 256, False, 1, False, 16),
    (4000, 4092, 132, 300, 6): (256, 256, False, 1, False, 16),
    (4100, 260, 1100, 20, 40): (32, 128, False, 1, False, 32),
    (8200, 68, 516, 9, 31): (32, 128, False, 1, False, 32),
}
