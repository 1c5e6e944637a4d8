"""Product shapes that the tests of large products run, with the tile (of
csrc/linear_plan.h: 0 is 64 x 64, 1 128 x 64, 2 128 x 128), the split and the
aligned copy that each gets: test_head_routes.py holds the plan to them, so that
a later rule cannot leave a kernel without a test."""

F32, BF16, F16 = "float32", "bfloat16", "float16"

# (M, N, K, type): tile, split, x and W copied to rows on 64-byte lines
FORWARD = {
    (4_099, 4_001, 72, F32): (2, False, False),
    (4_099, 4_001, 72, BF16): (2, False, True),
    (4_099, 4_001, 72, F16): (2, False, True),
    (2_051, 4_003, 40, BF16): (2, False, False),
    (2_051, 4_003, 40, F16): (2, False, False),
    (4_099, 600, 4_001, BF16): (2, True, False),
    (2_051, 4_003, 40, F32): (0, False, False),
}

# (M, N, K, type): tile and split of dx, of dW; x copied for dW
BACKWARD = {
    (600, 30_001, 513, BF16): (2, True, 2, False, False),
    (700, 20_001, 700, F16): (2, True, 2, False, False),
    (4_500, 300, 4_500, BF16): (2, False, 0, True, False),
    (4_099, 4_001, 72, BF16): (0, True, 0, True, True),
    (3_300, 3_203, 40, F16): (1, True, 0, True, True),
    # sums over words whose last 16 bytes of a row hold 5, 6 and 7 of 8 elements
    (600, 30_005, 513, BF16): (2, True, 2, False, False),
    (1_942, 15_182, 363, F16): (2, True, 0, False, True),
    (700, 20_007, 700, F16): (2, True, 2, False, False),
    (9_621, 5_518, 70, BF16): (2, True, 1, True, True),
    (47_089, 158, 87, BF16): (2, False, 0, True, False),
    (300, 4_100, 4_100, F32): (0, True, 2, False, False),
    (1_030, 9_001, 1_030, F32): (0, True, 1, False, False),
}
