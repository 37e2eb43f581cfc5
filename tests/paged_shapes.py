"""Batches and the kernels that they take: tiles of 32 rows (kg = 0), of 256 (kg = 1) or of 128 rows (kg = 2) for their long
sequences, with the keys cut or not.  tests/test_paged_plan_cpu.py holds the plan to what stands here, so that a change of its rules
does not move a batch to another kernel unseen."""

# name: kg, d, query heads, KV heads, lengths
PROMPTS = {f"{n}_d{d}": (kg, d, hq, hkv, lens) for d in (128, 64) for n, kg, hq, hkv, lens in [
    ("few", 0, 8, 2, [260, 17]),
    ("wide_even", 1, 32, 8, [130] * 16),
    ("wide_uneven", 1, 128, 16, [250, 1, 259, 17, 230]),
    ("wide_one_head", 1, 128, 128, [280, 256]),
    ("mid_two", 2, 32, 8, [700, 500]),
    ("mid_one", 2, 64, 8, [500]),
]}

# name: kg, joins, whether keys are cut indeed, d, query heads, KV heads, page size, lengths, new tokens
PAGES = {f"{n}_d{d}": (kg, joins, cut, d, hq, hkv, page, lens, new) for d in (128, 64)
         for n, kg, joins, cut, hq, hkv, page, lens, new in [
    ("few", 0, 1, True, 8, 2, 64, [6000, 5000, 300], [40, 33, 100]),
    ("token", 0, 1, True, 8, 2, 16, [3000, 40], [1, 1]),
    ("wide", 1, 0, False, 32, 8, 16, [150, 133] * 8, [100, 101] * 8),
    ("wide_cut", 1, 1, True, 32, 8, 16, [9000, 20000] + [100] * 20, [300, 1] + [80] * 20),
    # a chunk of more than 64 steps of 64 keys: pages are looked up a second and a third time
    ("wide_steps", 1, 1, False, 32, 8, 32, [9000], [1600]),
    ("mid", 2, 0, False, 8, 2, 16, [400] * 6, [350] * 6),
    ("mid_cut", 2, 1, True, 32, 8, 64, [9000, 1] + [100] * 8, [200, 1] + [60] * 8),
    # more than 64 steps of 128 keys
    ("mid_steps", 2, 1, False, 32, 8, 1024, [10000], [800]),
    # more new tokens than tokens: rows that see nothing beside ones that do
    ("wide_empty", 1, 0, False, 32, 8, 16, [60, 0, 90, 150] * 4, [100] * 16),
    ("mid_empty", 2, 0, False, 8, 2, 16, [100, 0, 300, 40, 7, 0], [350] * 6),
]}
