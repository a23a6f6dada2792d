"""Calls of paged_attn that between them take every kernel, and what each is planned to: name -> (lengths, rows of each sequence, page size,
K/V heads, query heads of each, head_dim, kernel as plans.PagedAttnPlan names it)."""
from plans import paged_plan

CALLS = {
    # paged_attn_split: one query tile, two, several groups of them; keys whole and cut
    "split_row": ([70, 200], [1, 1], 16, 2, 4, 128, "split"),
    "split_rows": ([300, 90], [150, 20], 16, 2, 1, 128, "split"),
    "split_heads_of_32": ([300, 40], [20, 30], 16, 2, 2, 32, "split"),
    "split_cut_row": ([1900, 40, 700], [1, 2, 1], 16, 2, 4, 128, "split+"),
    "split_cut_rows": ([1900, 500], [20, 33], 32, 2, 2, 64, "split+"),
    # blocks of 128 query rows, one group of wavefronts: keys whole, and cut
    "blocks": ([200, 90], [300, 20], 16, 8, 4, 128, "wide1"),
    "blocks_of_64": ([100, 333], [800, 60], 16, 8, 4, 64, "wide1"),
    "blocks_of_64_cut": ([8400], [100], 64, 2, 8, 64, "wide1+"),
    # two groups: each half of the keys, or each a block of its own (the shorter sequences of "shared"), and cut
    "halves": ([700, 333], [300, 40], 16, 8, 4, 128, "wide2"),
    "shared": ([700, 650, 550, 520], [320, 320, 320, 320], 32, 4, 8, 128, "wide2"),
    "halves_of_64": ([600], [800], 16, 8, 4, 64, "wide2"),
    "halves_cut": ([2600], [300], 16, 8, 4, 128, "wide2+"),
    "halves_cut_ragged": ([6500, 40, 2100], [100, 70, 129], 32, 2, 4, 128, "wide2+"),
}
BLOCKS = [name for name in CALLS if CALLS[name][6].startswith("wide")]


def plan_of(name, cache_dtype, dtype=0):
    """The plan of a call with a table one page wider than the longest sequence."""
    lens, counts, page, heads, group, dh, _ = CALLS[name]
    return paged_plan(heads * group, sum(counts), max(counts), dtype, len(lens), max(-(-n // page) for n in lens) + 1, page, heads, dh, cache_dtype)
