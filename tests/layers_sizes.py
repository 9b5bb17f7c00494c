"""Sizes of the layer tests that reach every kernel: the GPU tests run them, the CPU tests of the choices
(csrc/grad_choice.h, csrc/i8_choice.h) check that nothing is left out."""

# n_ids, rows, cols of an embedding gradient. In one launch; in windows; by sorted pairs, chunks of 8, 16,
# 32 and 64 tokens, joined at once or folded first; each with 4, 16 and 64 lanes to a row.
GRAD = [
    (3_900, 700, 20), (4_096, 300, 96), (1_000, 700, 515),
    (4_097, 50, 24), (600_000, 51, 3), (60_000, 100, 97), (20_000, 128, 1_000), (1_025, 3, 130),
    (20_000, 200, 24), (200_000, 5_000, 24), (1_100_000, 5_000, 8), (2_200_000, 400, 17),
    (9_000_000, 200_000, 8),
    (9_000, 2_000, 96), (100_000, 30_000, 96), (300_000, 200, 97), (600_000, 300_000, 96),
    (3, 43_000, 520), (4_000, 1_000, 520), (9_000, 400, 136), (8_192, 3_000, 4_096), (131_072, 9_000, 520),
    (4_400_000, 3_000, 136),
]

# m, n, k of an 8-bit product and the kernel that i8_choice.h takes for it: partial tiles in both directions,
# k short of a stage, of the stages in flight, and not a multiple of what shares it out.
SKINNY, TILE64, TILE128X64, TILE128_SPLIT, TILE128, TILE256, SHORT = range(7)
PRODUCTS = [
    (5, 3_001, 272, SKINNY), (40, 1_000, 8_208, SKINNY),
    (1_000, 1_001, 16, TILE64), (333, 1_030, 2_064, TILE64), (1_020, 1_020, 8_208, TILE64),
    (1_025, 1_030, 48, TILE128X64), (1_025, 1_030, 528, TILE128X64), (2_040, 1_003, 4_112, TILE128X64),
    (2_050, 1_030, 1_040, TILE128_SPLIT), (2_500, 1_501, 3_216, TILE128_SPLIT),
    (2_050, 1_030, 16, TILE128), (2_050, 1_030, 272, TILE128), (4_100, 1_030, 144, TILE128),
    (1_020, 8_187, 1_040, TILE128),
    (4_100, 1_030, 16, SHORT), (4_100, 1_030, 112, SHORT), (5_003, 2_001, 128, SHORT),
    (2_049, 8_190, 528, TILE256), (2_300, 8_193, 1_040, TILE256), (16_389, 1_300, 4_112, TILE256),
]

# Linear layers whose rows the kernel of few rows quantises itself, up to all of the LDS that it may take.
SKINNY_LINEAR = [(16, 640, 4_080), (13, 555, 5_021), (8, 300, 8_173), (1, 500, 65_520), (2, 16_001, 1_000)]
