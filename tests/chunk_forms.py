"""Calls on chunks, small enough for a comparison in 64 bits, that reach the forms which only large or many chunks take.  (Which form a call takes follows
from its shape by sqa_chunk_plan; test_chunk_forms.py holds that these still reach all of them.)  Test infrastructure only."""

TYPES = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]

# B, T, tokens before, Hq, Hkv, tokens of each sequence (None: all T)
ATTENTION = [
    # 128 rows of a workgroup, slots not shared out: many units
    (8, 150, [90] * 8, 64, 32, None), (32, 130, [0] * 32, 24, 8, [130 - 4 * b for b in range(32)]),
    (86, 129, [17 * b % 301 for b in range(86)], 3, 3, [129 - b for b in range(86)]),
    # ... the row tiles of 2, 4 and 8 units in turn, from an empty cache and behind some tokens
    (2, 2100, [0, 0], 8, 8, None), (4, 350, [5] * 4, 24, 8, None), (8, 129, [100] * 8, 64, 8, None), (32, 1024, [1] * 32, 2, 2, None),
    # ... not in turn: 40 units
    (5, 1025, [0] * 5, 8, 8, None),
    # ... and shared out among 2, 3 and more workgroups
    (3, 1025, [0] * 3, 8, 8, None), (2, 270, [1500] * 2, 32, 8, None), (4, 300, [3000] * 4, 8, 2, None), (1, 250, [4000], 8, 1, None),
    (3, 200, [2900, 1411, 0], 15, 3, [200, 199, 63]), (1, 257, [8200], 2, 1, None),
    # 64 rows of a workgroup: more slots than 32 rows are worth, or more units
    (40, 64, [200] * 40, 16, 16, None), (1, 512, [0], 32, 32, None), (2, 12, [2500, 2500], 40, 8, None), (5, 33, [1800, 7, 900, 0, 64], 20, 10, [33, 20, 33, 1, 32]),
]

# the same for scores: several row tiles of a workgroup, alone on its slots or one of those that share out the rows
SCORES = [
    (8, 300, [20] * 8, 32, 32, None), (3, 700, [2300] * 3, 24, 8, None), (16, 200, [100 * b for b in range(16)], 24, 8, [200 - 11 * b for b in range(16)]),
    (2, 1030, [0, 0], 16, 4, None), (1, 400, [4100], 64, 8, None), (4, 65, [1900] * 4, 40, 8, None), (1, 130, [16100], 16, 2, None),
    (5, 333, [1800, 7, 900, 0, 64], 20, 20, [333, 20, 330, 1, 129]),
]


def capacity(case):
    B, T, first, Hq, Hkv, n = case
    return max(f + m for f, m in zip(first, n or [T] * B)) + 1
