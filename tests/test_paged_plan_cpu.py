"""Which kernels batches take, and the device references of tests/paged_bounds.py against the numpy oracle."""
import numpy as np
import pytest

from oracle import paged_oracle as P
from tests import paged_bounds as B
from tests import paged_plan
from tests.paged_shapes import PAGES, PROMPTS


@pytest.mark.parametrize("name", PROMPTS)
def test_prompts_take_their_tiles(name):
    kg, d, hq, hkv, lens = PROMPTS[name]
    for extra in (0, 3):
        p = paged_plan.of_prompts("bf16", d, hq, hkv, lens, extra)
        assert p["kg"] == kg and p["joins"] == 0
    assert paged_plan.of_prompts("f32", d, hq, hkv, lens)["kg"] == 0


@pytest.mark.parametrize("name", PAGES)
def test_pages_take_their_tiles(name):
    kg, joins, _, d, hq, hkv, _, lens, new = PAGES[name]
    for extra in (0, 3):
        p = paged_plan.of_pages("bf16", d, hq, hkv, lens, new, extra)
        assert p["kg"] == kg and p["joins"] == joins


@pytest.mark.parametrize("n,m", [(5, 5), (3, 40), (7, 4), (4, 0), (1, 1)])
def test_device_reference_is_the_oracle(n, m):
    """Rows that see nothing, infinities and NaN among the values and a NaN key included."""
    rng = np.random.default_rng(n * 100 + m)
    q, k, v = (rng.standard_normal((x, 6)).astype(np.float32) for x in (n, m, m))
    for kind in ("finite", "values", "key"):
        if kind == "values" and m > 3:
            v[m - 2, 1], v[m // 2, 2], v[1, 2], v[0, 4] = np.nan, np.inf, -np.inf, np.inf
        if kind == "key" and m > 3:
            k[m - 2, 3] = np.nan
        for a, b in zip(B.attend_rows(q, k, v, 0.4, "cpu"), P.attend_rows(q, k, v, 0.4)):
            assert np.allclose(a, b, rtol=1e-12, atol=1e-14, equal_nan=True), kind


def test_sequences_of_padding_do_not_make_prompts_short():
    """Long prompts in a batch with room for many sequences take wide tiles, as they do alone."""
    for d in (128, 64):
        for lens, room in (([8192], 512), ([1024] * 4, 64), ([4000] + [30] * 70, 0), ([2048] * 2, 64)):
            assert paged_plan.of_prompts("bf16", d, 32, 8, lens + [0] * (room - len(lens)))["kg"] > 0, (d, lens[0], room)
        # prompts that are short indeed do not: what their tiles cost counts, not their number
        assert paged_plan.of_prompts("bf16", d, 8, 8, [60] * 8)["kg"] == 0
