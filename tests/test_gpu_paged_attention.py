"""Attention of new tokens over a paged cache against the float64 oracle.  Unused slots, pages and table entries hold NaN and
page numbers out of range in every test, and the workspace starts as garbage."""
import numpy as np
import pytest

from tests.paged_cases import Paged, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["heads", "tokens", "part"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(dtype, layout):
    from paper_2508_11661_amd import samkv as S
    Paged(1, dtype, 128, 8, 2, 16, [70, 1, 33], [1, 1, 5], extra_rows=2).check(S, layout)
    Paged(2, dtype, 64, 6, 2, 32, [300], [90]).check(S, layout)


@pytest.mark.parametrize("dtype,d,hq,hkv,page", [
    ("bf16", 128, 8, 2, 16), ("bf16", 64, 8, 2, 16), ("f32", 128, 8, 2, 16), ("f32", 64, 8, 2, 16),
    ("bf16", 128, 3, 3, 64), ("bf16", 64, 7, 1, 1024), ("f32", 64, 12, 1, 128), ("bf16", 128, 40, 1, 32),
    ("bf16", 128, 33, 1, 16), ("f32", 128, 33, 1, 512), ("bf16", 64, 16, 16, 256),
])
def test_single_tokens(dtype, d, hq, hkv, page):
    """Decoding: lengths around tiles of 32 and 64 keys, page ends and none at all."""
    from paper_2508_11661_amd import samkv as S
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 511, 513, 0, 700]
    Paged(3 + d, dtype, d, hq, hkv, page, lens, [1] * len(lens), uniform=True).check(S)


@pytest.mark.parametrize("dtype,d,hq,hkv,page,lens,new", [
    ("bf16", 128, 8, 2, 16, [40, 70, 200], [8, 9, 33]),           # 32, 36 and 132 rows per KV head
    ("bf16", 128, 4, 1, 32, [500, 64], [64, 64]),                 # the cache's end at a tile, and nothing but new tokens
    ("bf16", 64, 4, 1, 16, [300, 65, 33], [65, 65, 32]),
    ("bf16", 128, 6, 2, 64, [1000, 3, 400], [300, 3, 1]),         # three heads per KV head: tokens straddle waves
    ("bf16", 64, 14, 2, 16, [257, 129], [200, 37]),
    ("bf16", 128, 2, 2, 16, [600, 300], [513, 257]),
    ("bf16", 64, 2, 1, 128, [1500, 20], [129, 0]),
    ("bf16", 128, 32, 8, 16, [900, 333, 70], [100, 1, 64]),
    ("f32", 128, 8, 2, 16, [40, 70, 200], [8, 9, 33]),
    ("f32", 64, 6, 2, 32, [257, 64, 33], [64, 64, 1]),
    ("f32", 128, 2, 2, 16, [600, 300], [129, 257]),
    ("f32", 64, 32, 8, 64, [900, 333, 70], [40, 1, 64]),
])
def test_chunks(dtype, d, hq, hkv, page, lens, new):
    from paper_2508_11661_amd import samkv as S
    Paged(sum(lens) + d, dtype, d, hq, hkv, page, lens, new, extra_rows=1).check(S, "tokens")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_keys_and_empty_sequences(dtype):
    """More new tokens than tokens: the first ones have no slot (outputs 0, log-sum-exp -inf); sequences without tokens, without
    new tokens and without both; a padding sequence in a batch of one token each."""
    from paper_2508_11661_amd import samkv as S
    out, lse = Paged(5, dtype, 128, 8, 2, 16, [3, 0, 50, 0, 2], [7, 4, 0, 0, 2]).check(S)
    assert (out[:, :4] == 0).all() and np.isneginf(lse[:, :4]).all() and (out[:, 7:11] == 0).all()
    Paged(6, dtype, 64, 4, 4, 16, [0, 5, -3, 0], [1] * 4, uniform=True).check(S)
    Paged(7, dtype, 64, 4, 1, 16, [100, 40], [120, 60]).check(S)


@pytest.mark.parametrize("dtype,d,hq,hkv,lens", [
    ("bf16", 128, 4, 1, [9000]), ("bf16", 64, 8, 2, [20000, 5, 3000]), ("bf16", 128, 32, 8, [5000, 700, 1, 4097]),
    ("f32", 128, 4, 1, [6000, 40]), ("f32", 64, 8, 2, [9001]), ("bf16", 64, 1, 1, [40000]), ("bf16", 128, 130, 2, [3001, 9]),
])
def test_long_caches(dtype, d, hq, hkv, lens):
    """Keys cut into parts, beside short sequences that are not."""
    from paper_2508_11661_amd import samkv as S
    Paged(len(lens) + d, dtype, d, hq, hkv, 64, lens, [1] * len(lens)).check(S)
    Paged(len(lens) + d, dtype, d, hq, hkv, 16, lens, [min(3, n) for n in lens]).check(S)


def test_many_sequences():
    from paper_2508_11661_amd import samkv as S
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 90, 300)]
    Paged(8, "bf16", 64, 4, 2, 16, lens, [1] * 300, uniform=True).check(S)
    new = [int(min(n, x)) for n, x in zip(lens, rng.integers(0, 9, 300))]
    Paged(9, "bf16", 128, 4, 2, 16, lens, new, extra_rows=5).check(S)
    Paged(9, "f32", 64, 4, 2, 16, lens, new, extra_rows=5).check(S)


@pytest.mark.parametrize("dtype,d,hq,hkv,lens,new", [
    ("bf16", 128, 4, 1, [300, 90], [150, 90]), ("bf16", 64, 2, 2, [700], [600]), ("f32", 128, 4, 2, [130, 70], [60, 70]),
    ("bf16", 128, 8, 2, [100], [8]), ("f32", 64, 3, 1, [65], [33]),
])
def test_later_tokens_do_not_reach_a_row(dtype, d, hq, hkv, lens, new):
    """Infinities and NaN in the keys and values of new tokens: rows before them come out as if they were not there, and rows
    that see them as the definition has it."""
    from paper_2508_11661_amd import samkv as S
    x = Paged(11 + d, dtype, d, hq, hkv, 16, lens, new)
    clean, clean_lse = x.attend(S)
    s, n = 0, new[0]
    slots = [lens[0] - 2, lens[0] - n // 2, lens[0] - n + 1]
    for slot, (value, ch) in zip(slots, [(np.nan, 3), (np.inf, d - 1), (-np.inf, 0)]):
        x.v[x.table[s, slot // 16], :, slot % 16, ch] = value
    out, lse = x.attend(S)
    # Rows that meet such values may be computed by other sums than before (each within the bound of check(), so the two runs
    # are within twice that of each other): what is finite is held to the oracle, not to the bits of the clean run.
    ref = x.oracle()
    assert (~np.isfinite(ref.out)).any()
    check(out, lse, ref, d, x.scale, dtype, "with infinities and NaN among the values")
    x = Paged(11 + d, dtype, d, hq, hkv, 16, lens, new)
    slot = lens[0] - n // 2
    x.k[x.table[s, slot // 16], :, slot % 16, 5] = np.nan
    out, lse = x.attend(S)
    before, after = slice(0, n - n // 2), slice(n - n // 2, n)
    assert np.array_equal(out[:, before], clean[:, before]) and np.array_equal(lse[:, before], clean_lse[:, before])
    assert np.isnan(out[:, after]).all() and np.array_equal(out[:, n:], clean[:, n:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_beyond_bounds_stay_inside(dtype):
    """Lengths above max_len and below zero, prefix sums that run past the rows or backwards, more new tokens than max_new."""
    from paper_2508_11661_amd import samkv as S
    x = Paged(12, dtype, 64, 4, 2, 16, [60, 60, 60], [4, 4, 4])
    x.max_len, x.max_new = 50, 3
    x.lens = [1000000, -5, 20]
    x.check(S)
    x = Paged(13, dtype, 64, 4, 2, 16, [60, 60, 60], [4, 4, 4])
    x.cu = np.array([-3, 2, 2, 1 << 30], np.int32)   # rows 0 and 1, none, 2 to 11, of which max_new = 4 count
    x.check(S)
    x.cu = np.array([3, 1, 5, 8], np.int32)          # none (backwards), 1 to 4, 5 to 7
    x.check(S)


def test_scores_of_all_sizes():
    """Running maxima that rise and fall by far more than 2^8, and rows whose weights all sit on one key."""
    from paper_2508_11661_amd import samkv as S
    for dtype, new in (("bf16", 1), ("bf16", 80), ("f32", 5)):
        x = Paged(14, dtype, 128, 4, 1, 16, [700], [new])
        ramp = np.float32(2.0) ** np.random.default_rng(3).integers(-6, 4, 700).astype(np.float32)
        slots = np.arange(700)
        x.k[x.table[0, slots // 16], :, slots % 16] *= ramp[:, None, None]
        x.check(S)


def test_lse_may_be_left_out_and_runs_repeat():
    from paper_2508_11661_amd import samkv as S
    x = Paged(15, "bf16", 128, 8, 2, 16, [5000, 300], [1, 200])
    a, l = x.attend(S)
    b, untouched = x.attend(S, with_lse=False)
    c, l2 = x.attend(S)
    assert np.array_equal(a, b) and np.array_equal(a, c) and np.array_equal(l, l2) and (untouched == 7.0).all()


def test_pages_beyond_32_bits():
    """A cache of more than 4 GB per tensor: pages at its end."""
    import torch
    from paper_2508_11661_amd import samkv as S
    n_pages, hkv, page, d = (5 << 30) // (2 * 64 * 128 * 2), 2, 64, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    small = torch.randn((4, hkv, page, d), device="cuda", generator=gen).to(torch.bfloat16)
    k, v = (torch.empty((n_pages, hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.randn((8, 1, d), device="cuda", generator=gen).to(torch.bfloat16)
    far = torch.tensor([n_pages - 1, n_pages // 2, n_pages - 2, 0], device="cuda")
    k[far], v[far] = small, small.flip(0)
    outs = []
    for cache, table in ((S.PagedCache(k, v), far), (S.PagedCache(small, small.flip(0).contiguous()), torch.arange(4, device="cuda"))):
        batch = S.PagedBatch(table.to(torch.int32)[None], torch.tensor([250], dtype=torch.int32, device="cuda"), 250)
        out, lse = torch.empty_like(q), torch.empty((8, 1), device="cuda")
        ws = torch.empty((S.samkv_paged_workspace_bytes(cache, batch, 8),), dtype=torch.uint8, device="cuda")
        S.samkv_paged_append(cache, batch, small[0, :, 5:6], small[1, :, 6:7])
        S.samkv_paged_attn(cache, batch, q, d ** -0.5, out, lse, ws)
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
