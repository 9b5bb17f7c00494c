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
