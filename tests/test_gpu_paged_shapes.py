"""Batches that take wide tiles: many sequences, chunks, mixtures of long and short ones, over prompts and over pages."""
import numpy as np
import pytest

from oracle import paged_oracle as P
from tests.paged_cases import Paged, check
from tests.test_gpu_prefill_attention import _case, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,hq,hkv,page,lens,new", [
    # more sequences than a wave has lanes, one of them with many rows: tiles of 256 and of 128 rows
    ("bf16", 128, 32, 8, 16, [1500] + [50 + 2 * i for i in range(69)], [1000] + [8] * 69),
    ("bf16", 64, 32, 8, 32, [1500] + [50 + 2 * i for i in range(69)], [1000] + [8] * 69),
    ("bf16", 128, 8, 2, 64, [20 + 3 * i for i in range(90)], [0, 1, 40, 7, 12, 3] * 15),
    ("bf16", 64, 8, 2, 16, [20 + 3 * i for i in range(90)], [0, 1, 40, 7, 12, 3] * 15),
    # the keys of wide tiles cut into chunks, beside sequences of one token
    ("bf16", 128, 32, 8, 16, [2600, 700, 1], [1540, 1, 1]),
    ("bf16", 64, 32, 8, 16, [2600, 700, 1], [1540, 1, 1]),
    ("bf16", 128, 8, 2, 16, [6000, 5000, 300], [40, 33, 100]),
    ("bf16", 64, 8, 2, 1024, [6000, 5000, 300], [40, 33, 100]),
    ("bf16", 128, 4, 1, 16, [9000] + [30] * 70, [200] + [1] * 70),
    # as many rows per KV head as two tiles of 32 hold, and more
    ("bf16", 128, 8, 2, 16, [4000, 900], [16, 16]),
    ("bf16", 128, 8, 2, 16, [4000, 900], [17, 16]),
    ("f32", 64, 4, 2, 16, [3001] + [20] * 80, [2] + [1] * 80),
])
def test_pages(dtype, d, hq, hkv, page, lens, new):
    from paper_2508_11661_amd import samkv as S
    Paged(len(lens) + d, dtype, d, hq, hkv, page, lens, new).check(S, "tokens")


@pytest.mark.parametrize("d,hq,hkv,page,lens,new", [
    (128, 8, 2, 16, [400] * 6, [350] * 6), (64, 8, 2, 32, [400] * 6, [350] * 6),                       # more than 512 tiles of 32 rows
    (128, 6, 2, 64, [300, 80] * 40, [100, 40] * 40), (64, 6, 2, 64, [300, 80] * 40, [100, 40] * 40),  # and more than 64 sequences
    (128, 8, 2, 16, [6000, 5000, 300, 2], [60, 50, 100, 1]), (64, 8, 2, 16, [9000, 5000, 300, 2], [120, 100, 100, 1]),  # long ones
    (128, 16, 1, 1024, [7000, 10], [100, 10]),
])
def test_pages_in_tiles_of_128_rows(d, hq, hkv, page, lens, new):
    from paper_2508_11661_amd import samkv as S
    Paged(sum(new) + d, "bf16", d, hq, hkv, page, lens, new, extra_rows=2).check(S, "tokens")


@pytest.mark.parametrize("d,hq,hkv,lens", [
    (128, 32, 8, [700, 1, 300] + [30] * 70), (64, 32, 8, [700, 1, 300] + [30] * 70), (128, 32, 8, [520] * 6), (64, 32, 8, [520] * 12),
    (128, 16, 2, [1400]), (64, 16, 2, [2100]), (128, 5, 1, [257, 256, 255, 9, 8, 7]),
])
def test_prompts(d, hq, hkv, lens):
    (q, k, v), cu = _case(sum(lens) + d, "bf16", d, hq, hkv, lens, extra=2)
    ref = P.prefill(q, k, v, cu, max(lens), d ** -0.5)
    out, lse = _run("bf16", q, k, v, cu, max(lens), d ** -0.5, "tokens")
    check(out, lse, ref, d, d ** -0.5, "bf16", f"prompts d={d} {lens[:4]}")
    assert (out[:, ~ref.written] == 7.0).all() and (lse[:, ~ref.written] == 7.0).all()


def test_padding_sequences():
    """A table with room for many more sequences than there are new tokens."""
    from paper_2508_11661_amd import samkv as S
    Paged(31, "bf16", 128, 8, 2, 16, [0] * 200 + [900] + [0] * 300, [0] * 200 + [1] + [0] * 300).check(S)
    Paged(32, "bf16", 128, 8, 2, 16, [0] * 100 + [900] + [0] * 30, [0] * 100 + [150] + [0] * 30).check(S)
