"""Sizes of the 8-bit linear, each with the kernel that it is there for: at least one ragged size for every kernel that
w8a8_linear can launch.  test_w8_host.py holds them to the plan, test_gpu_w8.py runs them.
"""

# (tokens, output features, input features, kernel, parts of K): rows kernels as row tiles x token tiles x waves, the others
# as their tiles of output features x tokens
CASES = [
    (1, 16403, 1088, "rows 1x1x8", 1), (3, 28679, 2112, "rows 1x1x8", 1),
    (9, 2050, 1088, "rows 1x1x4", 1), (16, 130, 8192, "rows 1x1x4", 1),
    (16, 9001, 1088, "rows 2x1x4", 1), (3, 16003, 704, "rows 2x1x4", 1),
    (31, 1027, 704, "rows 1x2x4", 1), (17, 515, 2112, "rows 1x2x4", 1),
    (31, 4099, 2112, "rows 2x2x4", 1), (17, 6001, 192, "rows 2x2x4", 1),
    (17, 12805, 1088, "rows 4x2x4", 1), (24, 9001, 704, "rows 4x2x4", 1),
    (16, 16403, 1088, "128x32", 1), (31, 16003, 8256, "128x32", 1), (24, 28679, 1088, "128x32", 1),
    (17, 4099, 11008, "128x32", 4), (16, 1027, 11008, "128x32", 15),
    (1500, 1027, 704, "128x64", 1), (513, 2050, 2112, "128x64", 1), (777, 1027, 8256, "128x64", 2), (33, 1027, 14336, "128x64", 16),
    (1500, 4099, 704, "256x128", 1), (2049, 1027, 4160, "256x128", 1), (333, 16003, 2112, "256x128", 1),
    (129, 6001, 8192, "256x128", 5), (1000, 1027, 11008, "256x128", 6),
    (1000, 16003, 320, "256x256", 1), (777, 16003, 1088, "256x256", 1), (1500, 6001, 4160, "256x256", 1),
    (1000, 4099, 8192, "256x256", 3), (2300, 1027, 11008, "256x256", 5),
]
ROWS = ("1x1x8", "1x1x4", "2x1x4", "1x2x4", "2x2x4", "4x2x4")
TILES = ("128x32", "128x64", "256x128", "256x256")
