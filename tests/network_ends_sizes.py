"""Sizes of the vocabulary loss that the GPU tests run: T, d, V, entries between rows, entries before the first.
Few rows, few tiles, each tile; odd rows; a vocabulary below and above a tile; several pieces."""
HEAD = [(1, 1, 1, 0, 0), (1, 4096, 1000, 0, 0), (2, 64, 33, 0, 0), (5, 7, 3, 0, 0), (17, 131, 257, 1, 1), (16, 1001, 700, 0, 0),
        (33, 1024, 100, 0, 0), (33, 72, 1000, 8, 8), (70, 130, 65, 3, 1), (200, 264, 2000, 0, 0), (129, 520, 4100, 0, 0),
        (600, 72, 9001, 0, 0), (300, 1000, 515, 0, 2), (64, 96, 300, 0, 0), (65, 96, 300, 0, 0),
        (32, 72, 20000, 0, 0), (9, 131, 17001, 3, 1), (4, 200, 9000, 0, 0)]
# With references on the GPU: tiles of 256, pieces, parts of the summed axis, x as columns
HEAD_LARGE = [(2100, 520, 33000, 0, 0), (4200, 136, 40003, 1, 3), (1030, 264, 70000, 0, 0), (3000, 512, 600, 0, 0), (9000, 72, 9000, 0, 0),
              (2048, 1024, 16384, 0, 0), (5000, 2560, 14000, 0, 0)]
