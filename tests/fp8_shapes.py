"""Shapes of the 8-bit product that take each of its tiles on 256 compute units
(csrc/linear_fp8_tiles.h), in at most one round of workgroups and in more, with
ragged rows, columns and last blocks of k.  A host test checks the tiles; the GPU
tests run the shapes."""

# (rows, columns, groups of waves)
TILES = {"bf16": [(256, 256, 1), (192, 256, 1), (128, 256, 1), (128, 128, 1), (64, 128, 1), (64, 64, 1), (64, 64, 2),
                  (192, 192, 1), (64, 128, 2)],
         "fp32": [(256, 128, 1), (128, 128, 2), (64, 64, 1), (64, 64, 2), (192, 192, 1)]}

# (output type, tile, more than one round, M, N, K)
SHAPES = [
    ("bf16", 0, False, 12391, 776, 272),
    ("bf16", 0, True, 11575, 2480, 80),
    ("bf16", 1, False, 13209, 584, 80),
    ("bf16", 1, True, 9910, 1744, 80),
    ("bf16", 2, False, 321, 10920, 656),
    ("bf16", 2, True, 10809, 1288, 272),
    ("bf16", 3, False, 145, 10888, 656),
    ("bf16", 3, True, 12439, 600, 80),
    ("bf16", 4, False, 67, 72, 656),
    ("bf16", 4, True, 265, 10952, 272),
    ("bf16", 5, False, 67, 16, 272),
    ("bf16", 5, True, 521, 7184, 80),
    ("bf16", 6, False, 67, 72, 2064),
    ("bf16", 6, False, 1561, 520, 4240),
    ("bf16", 7, False, 11748, 520, 80),
    ("bf16", 7, False, 1561, 5000, 1040),
    ("bf16", 7, True, 8229, 1824, 80),
    ("bf16", 8, False, 1895, 840, 4240),
    ("bf16", 8, False, 6459, 200, 4112),
    ("bf16", 8, True, 289, 10912, 4240),
    ("fp32", 0, False, 321, 10888, 272),
    ("fp32", 0, True, 1291, 8880, 272),
    ("fp32", 1, False, 145, 10888, 656),
    ("fp32", 1, True, 10231, 848, 80),
    ("fp32", 1, False, 3001, 1000, 1936),
    ("fp32", 2, False, 67, 16, 80),
    ("fp32", 2, True, 10889, 264, 272),
    ("fp32", 3, False, 67, 16, 656),
    ("fp32", 3, False, 261, 1928, 2064),
    ("fp32", 4, False, 1561, 5000, 1040),
    ("fp32", 4, True, 1037, 10952, 80),
]
