"""Shapes of the tests of attention over shared prefixes: B, Bp, H, H_kv, N, P, N_k,
layout, left, right, q_len, p_len, k_len."""

CASES = [
    # one sequence, one key each; a prefix alone; an empty suffix
    (1, 1, 1, 1, 1, 1, 1, "bhnd", -1, -1, None, None, None),
    (3, 1, 2, 2, 1, 70, 0, "bhnd", -1, 0, None, None, None),
    (2, 2, 2, 1, 5, 33, 0, "bnhd", -1, -1, None, [33, 1], None),
    # single tokens of sequences that share prefixes, short ones and long ones
    (4, 1, 6, 6, 1, 196, 16, "bhnd", -1, -1, None, None, None),
    (6, 2, 8, 2, 1, 1700, 40, "bnhd", -1, 0, None, [1700, 129], [40, 0, 1, 17, 32, 33]),
    (40, 1, 4, 1, 1, 1500, 100, "bnhd", -1, 0, None, None, [100 - 2 * i for i in range(40)]),
    (36, 3, 12, 4, 1, 1300, 65, "bhnd", -1, 0, None, [1300, 0, 257], None),
    (24, 1, 8, 8, 2, 3000, 1100, "bnhd", -1, 0, None, [2999], [1100 - 40 * i for i in range(24)]),
    (5, 1, 32, 1, 1, 6640, 77, "bhnd", -1, 0, [1, 0, 1, 1, 1], None, [77, 5, 0, 1, 64]),
    (3, 1, 2, 2, 1, 1100, 0, "bhnd", -1, 0, None, [1040], None),
    (5, 1, 8, 4, 3, 1640, 77, "bnhd", -1, 0, [3, 0, 1, 2, 3], None, [77, 5, 0, 1, 64]),
    # many prefixes, whose keys are not split
    (24, 12, 12, 12, 1, 1030, 9, "bnhd", -1, 0, None, [1030 - 90 * i for i in range(12)], None),
    (297, 9, 16, 16, 1, 1030, 3, "bhnd", -1, 0, None, [1030 - 100 * i for i in range(9)], None),
    # keys and values of 64 MB and more: with sharing (few rows and many), and without
    (12, 1, 8, 8, 1, 40000, 2000, "bnhd", -1, 0, None, [39999], [2000 - 150 * i for i in range(12)]),
    (140, 2, 16, 8, 1, 9000, 400, "bhnd", -1, 0, None, [9000, 8191], [400 - 2 * i for i in range(140)]),
    (3, 3, 8, 8, 1, 30000, 700, "bhnd", -1, 0, None, [30000, 1, 0], [700, 0, 65]),
    # windows that hide some, or all, of a prefix, or reach over its end
    (8, 2, 4, 2, 2, 500, 200, "bnhd", 230, 0, None, [500, 400], [200, 10, 0, 199, 100, 3, 2, 1]),
    (8, 2, 4, 2, 2, 1500, 200, "bnhd", 230, 0, None, [1500, 400], [200, 10, 0, 199, 100, 3, 2, 1]),
    (70, 1, 2, 1, 1, 1200, 300, "bhnd", 700, 2, None, None, [300 - 4 * i for i in range(70)]),
    (7, 1, 4, 1, 4, 260, 90, "bhnd", 40, 3, None, None, [90, 60, 41, 40, 39, 4, 0]),
    (4, 1, 2, 2, 1, 400, 300, "bhnd", 0, 0, None, None, [300, 1, 0, 299]),
    # queries in front of their first key, and of the prefix
    (3, 1, 4, 2, 9, 5, 3, "bnhd", -1, 0, None, None, [3, 0, 1]),
    (4, 2, 2, 1, 50, 20, 10, "bhnd", -1, 0, [50, 20, 31, 1], [20, 0], [10, 0, 10, 0]),
    # prompts behind a prefix
    (2, 1, 4, 2, 150, 333, 150, "bnhd", -1, 0, [150, 77], None, [150, 77]),
    (3, 1, 6, 2, 70, 500, 70, "bhnd", -1, 0, [70, 1, 0], [499], [70, 1, 0]),
    (2, 2, 2, 2, 260, 129, 260, "bhnd", 100, 0, None, [129, 64], None),
    (2, 1, 2, 1, 130, 1, 400, "bnhd", -1, -1, None, None, [400, 1]),
    (1, 1, 2, 2, 300, 2000, 300, "bnhd", -1, 0, None, None, None),
    (66, 2, 4, 4, 129, 90, 70, "bnhd", -1, 0, None, [90, 31], None),
    (16, 1, 16, 16, 200, 65, 200, "bhnd", 70, 5, [200 - 13 * i for i in range(16)], None, [200 - 13 * i for i in range(16)]),
    # enough keys for tiles of 128 rows: without splits, and with them
    (32, 1, 8, 8, 256, 1500, 500, "bnhd", -1, 0, None, [1437], [500 - 15 * i for i in range(32)]),
    (3, 1, 32, 32, 300, 4000, 300, "bnhd", -1, 0, [300, 100, 0], [3937], [300, 100, 255]),
    (3, 1, 32, 16, 150, 4100, 700, "bhnd", 3900, 40, None, None, [700, 0, 65]),
]
