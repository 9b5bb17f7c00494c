"""Sizes that reach every kernel of the 4-bit products and of the block norms: the GPU tests run them, the CPU
tests of the choices (csrc/mx_choice.h, csrc/norm_choice.h) check that nothing is left out."""

# m, n, k of a 4-bit product and the kernel that mx_choice.h takes for it: partial tiles in both directions,
# k of less than a stage, of one, of half a stage more, of two stages and more than are on the way.
SKINNY, TILE64, TILE128, TILE256 = range(4)
PRODUCTS = [
    (5, 3_001, 640, SKINNY), (40, 1_000, 8_320, SKINNY), (17, 4_096, 5_000, SKINNY),
    (1_000, 1_001, 128, TILE64), (333, 1_030, 2_055, TILE64), (1_020, 2_047, 256, TILE64),
    (700, 900, 384, TILE64), (600, 777, 512, TILE64), (65, 4_100, 1_664, TILE64), (800, 1_000, 9_000, TILE64),
    (4_100, 1_030, 96, TILE128), (2_050, 1_200, 256, TILE128), (2_100, 1_281, 384, TILE128),
    (300, 9_001, 640, TILE128), (50_000, 65, 300, TILE128), (2_300, 3_300, 2_176, TILE128),
    (3_000, 3_001, 128, TILE256), (2_999, 3_100, 256, TILE256), (4_003, 2_500, 384, TILE256),
    (2_049, 4_290, 1_152, TILE256), (10_000, 1_000, 4_224, TILE256), (16_389, 5_001, 4_096, TILE256),
]

# Linear layers whose rows the skinny kernel puts in 4 bits itself, and some just past its limits.
INSIDE = [(1, 500, 32_768), (16, 640, 2_048), (13, 555, 2_400), (1, 16_384, 4_096), (7, 300, 4_600),
          (2, 9_000, 99)]
OUTSIDE = [(1, 500, 32_769), (16, 640, 2_049), (1, 16_400, 96), (17, 64, 96), (16, 4_097, 2_048)]

# Rows and columns of the norms: one column; part of a block of 8; rows for 16 lanes to 1,024, wavefronts that
# are no power of two among them; odd ends and whole blocks of each; rows in pieces.
NORMS = [(1, 1), (3, 2), (5, 7), (70, 8), (33, 97), (40, 128), (37, 136), (29, 253), (21, 256), (19, 300),
         (18, 512), (9, 520), (11, 1_003), (7, 1_024), (5, 1_032), (5, 1_113), (6, 2_047), (6, 2_048), (5, 2_051),
         (4, 2_344), (4, 4_096), (3, 4_101), (3, 4_104), (3, 5_000), (3, 6_093), (3, 8_192), (2, 9_001), (2, 9_680),
         (2, 16_384), (2, 16_392), (3, 20_003), (2, 40_000)]

# More rows than a launch has groups of lanes, several times.
MANY_ROWS = [(17_000, 96), (9_000, 200), (5_000, 500), (9_000, 520), (2_700, 1_300), (2_100, 2_048),
             (700, 4_096), (600, 8_192)]
