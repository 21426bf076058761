"""Cases that reach each form of the paged dense attention: 1 (few rows), 2, 4 and 8 waves, whole tiles and split keys,
pages of at least 64 rows and smaller ones, and runs of sub-blocks longer than a window of page places."""
from __future__ import annotations

import ctypes

from paper_2606_13392_amd import msa

# name, waves, keys split, q_rows, kv_lens, H_q, H_kv, page, rows behind the last sequence
VARIANTS = [
    ("two_waves", 2, False, [8, 5, 1], [70, 300, 33], 16, 2, 64, 1),
    ("two_waves_16", 2, False, [7, 0, 8], [7, 130, 201], 16, 2, 16, 0),
    ("two_waves_split", 2, True, [8], [3000], 16, 2, 128, 0),
    ("two_waves_split_32", 2, True, [6, 8, 1], [2500, 1000, 4000], 8, 1, 32, 2),
    ("two_waves_split_group_of_16", 2, True, [3, 4], [1800, 3500], 32, 2, 16, 0),
    ("two_waves_split_group_of_3", 2, True, [20, 11], [900, 2000], 6, 2, 64, 0),
    ("two_waves_group_of_1", 2, False, [64], [64], 4, 4, 32, 0),
    ("four_waves", 4, False, [13], [400], 16, 2, 64, 0),
    ("four_waves_16", 4, False, [16, 9], [100, 220], 16, 2, 16, 0),
    ("four_waves_split_16", 4, True, [12, 16], [2500, 4100], 16, 2, 16, 0),
    ("four_waves_split", 4, True, [16, 1], [2000, 3000], 16, 2, 64, 1),
    ("four_waves_split_32", 4, True, [10], [3000], 8, 1, 32, 3),
    ("eight_waves_32", 8, False, [100], [300], 16, 2, 32, 0),
    ("eight_waves_split_16", 8, True, [33, 50], [3000, 2000], 8, 1, 16, 0),
    ("few_rows_16", 1, False, [4, 1], [65, 400], 16, 2, 16, 0),
    ("few_rows_split_16", 1, True, [1], [5000], 16, 2, 16, 0),
    ("few_rows_split_32", 1, True, [1, 4, 2], [3000, 4097, 50], 8, 1, 32, 1),
]

# the same; a CTA's run of one tile crosses a window of 64 page places at least twice (a window holds 64 sub-blocks on
# pages of 64 rows and more, 32 and 16 on pages of 32 and 16), where the keys are split from a sub-block that is no
# multiple of the window.  More than 256 sequences are never split.
LONG = [
    ("few_rows_64", 1, True, [1], [51300], 64, 64, 64, 0),
    ("few_rows_16", 1, True, [1, 1], [9000, 3000], 64, 64, 16, 0),
    ("few_rows_32", 1, True, [2], [17100], 128, 64, 32, 0),
    ("eight_waves_64", 8, True, [150], [36000], 64, 64, 64, 0),
    ("eight_waves_16", 8, True, [150], [9000], 64, 64, 16, 0),
    ("four_waves_16", 4, True, [100], [18000], 64, 64, 16, 0),
    ("two_waves_32", 2, True, [40], [34100], 64, 64, 32, 0),
    ("few_rows_whole_64", 1, False, [1] * 257, [9000] + [1 + i for i in range(256)], 8, 1, 64, 0),
    ("few_rows_whole_16", 1, False, [1] * 257, [1 + i for i in range(256)] + [9001], 8, 1, 16, 0),
    ("eight_waves_whole_64", 8, False, [1] * 256 + [40], [5] * 256 + [9050], 8, 1, 128, 0),
    ("two_waves_whole_16", 2, False, [8] + [1] * 256, [2500] + [5] * 256, 8, 1, 16, 0),
]


def workspace(q_rows, kv_lens, H_q, H_kv, page, pad=0):
    total = sum(-(-n // page) for n in kv_lens) * page
    c = msa.MsaSeqsC(len(q_rows), sum(q_rows), total, max(q_rows), max(kv_lens), 8, 8, 8, 8, -(-max(kv_lens) // page), page)
    return msa.lib().msa_dense_attn_paged_workspace_size(ctypes.byref(c), H_q, H_kv, 128)


def waves_of(rows, group):
    """Waves per tile for calls of up to ``rows`` rows per sequence (up to a tile of 8 waves), told from workspace sizes:
    parts of 2 tiles of 32 * waves rows for each of 512 CTAs (2 and 4 waves) or 256 (1 and 8)."""
    rows = min(rows, 8 * (32 // group))
    part = 4 * 2 * 32 * 129
    size = workspace([rows], [65536], group, 1, 64)
    if size != 2048 * part:
        return {256 * part: 1, 1024 * part: 2}[size]
    # two tiles for each of 64 groups and 13 sub-blocks: 128 of 512 CTAs (split) or of 256 (not)
    return 4 if workspace([rows, rows], [13 * 64] * 2, group * 64, 64, 64) else 8


def run_length(case):
    """(sub-blocks of the longest run of a CTA in one tile, sub-blocks per window)."""
    name, waves, split, q_rows, kv_lens, H_q, H_kv, page, pad = case
    qt = waves * (32 // (H_q // H_kv))
    blocks = [-(-n // 64) for n in kv_lens]
    longest = max(blocks)
    if split:
        ctas = (256 if waves in (1, 8) else 512) // H_kv
        longest = min(longest, max(4, -(-sum(-(-q // qt) * b for q, b in zip(q_rows, blocks)) // ctas)))
    return longest, min(page, 64)
