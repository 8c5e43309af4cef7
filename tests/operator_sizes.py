"""Sizes that take certain tiles on 256 CUs: run by test_gpu_operators_tiles.py, held to their
tiles by test_operator_plans.py."""

# T, n, m of the product with codes, one scale a row: 256 x 256 tiles over 3, 5, 7 and 8 chunks of 128 codes
LINEAR_BIG = [(2003, 631, 8150), (1990, 900, 8190), (2003, 384, 8150), (2048, 871, 8192)]

# T, d, f of the gated product: 256 x 256 tiles over 5, 7, 6 (of rows that are padded first) and 18 chunks
GATED = [(2003, 320, 4075), (2003, 440, 4075), (2003, 333, 4075), (1999, 1104, 4080)]

# T, d, f, dx, dw of the gradients, then the (tile, parts) of dx and of dw
BACKWARD = [
    (2003, 440, 4075, True, True, (128, 4), (128, 1)),     # dG and dU from 256 x 256 tiles
    (4000, 4040, 300, True, False, (256, 1), None),        # 10 chunks, in two pieces of 5
    (300, 4040, 2000, False, True, None, (256, 1)),        # 5 chunks, the last of 44 tokens
    (12000, 1000, 2000, True, True, (256, 1), (256, 4)),
    (4100, 1990, 6000, True, False, (256, 3), None),       # a part holds the end of one piece and the next's start
    (60, 4040, 4000, False, True, None, (256, 1)),         # x once more, beside the rests of dG and dU
    (1111, 1000, 2731, True, True, (128, 3), (128, 1)),
]
