"""Dense attention calls that take the 128-row kernel, whole and with split keys
(tests/test_dense_plans.py checks that they do)."""

RAGGED = [140, 77, 0, 1, 128, 129, 140, 33]
TILE_CASES = [
    # B, H, Hk, N, Nk, layout, left, right, q_len, k_len
    (8, 16, 16, 130, 130, "qkv", -1, -1, None, None),              # a last tile of two rows: waves without rows
    (5, 12, 4, 521, 521, "bnhd", -1, 0, [521, 400, 1, 0, 130], [521, 400, 1, 0, 130]),
    (5, 12, 4, 521, 521, "bhnd", -1, 0, None, None),
    (8, 16, 16, 257, 257, "bhnd", 40, 7, None, None),
    (8, 16, 16, 200, 300, "bhnd", 30, -1, None, None),
    (8, 16, 16, 300, 150, "bhnd", -1, 0, None, None),              # the first queries see nothing
    (8, 16, 16, 140, 1100, "bhnd", -1, 0, None, None),             # new queries behind a prefix, keys split
    (8, 16, 16, 140, 1100, "bnhd", -1, -1, RAGGED, [1100, 513, 0, 1, 64, 1027, 0, 700]),
    (8, 16, 16, 129, 2048, "bnhd", 1500, 0, None, [2048, 1, 0, 2047, 1000, 130, 1536, 64]),
    (1, 6, 2, 5600, 90, "bhnd", -1, -1, None, None),               # many rows of few keys
]
