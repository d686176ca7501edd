"""Sizes at which a workgroup of the class losses' kernels streams several tiles, so that their loops turn: (T, V, D) by what holds
and what streams.  test_class_tiles.py checks the counts against the plan, test_gpu_class_tiles.py runs them."""

# many rows and many classes: four waves beside each other in both directions; tables that are laid out first and, in 16 bits at a
# whole depth, as they are
BOTH = [(2100, 9000, 64), (2100, 9000, 50), (2100, 9000, 128), (2100, 9001, 100), (1500, 9000, 256), (1500, 9000, 200)]
# few rows past a large table: waves of a workgroup share the streamed classes
FEW_ROWS = [(70, 100_003, 64), (70, 100_003, 100), (70, 100_003, 256), (20, 200_001, 64), (20, 200_001, 128), (20, 200_001, 200)]
# many rows past few classes: they share the streamed rows in the gradient
FEW_CLASSES = [(60_001, 60, 64), (60_001, 60, 100), (60_001, 60, 200), (40_003, 30, 40), (40_003, 30, 128), (40_003, 30, 256)]
# rows of more than 256 elements
WIDE = [(300, 9000, 384), (300, 9001, 300), (300, 9000, 602), (200, 6001, 1024)]
