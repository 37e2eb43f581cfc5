"""What the device makes of a batch's lengths stays within the grid and the workspace that the host made from its bounds: a tile whose
partial results had no slot would not be computed."""
import random

import pytest

from tests import paged_plan


def _holds(dtype, d, hq, hkv, lens, new, max_len=None, room=0):
    n_rows = sum(new) + room
    if n_rows < 1 or hq * n_rows >= 1 << 27:
        return None
    max_len = max(max(lens), 1) if max_len is None else max_len
    p = paged_plan.plan(dtype, d, hq, hkv, len(lens), n_rows, max(max(new), 1), max_len, True)
    items, slots = paged_plan.items(p["kg"], p, hq, hkv, lens, new)
    assert items <= p["max_items"] and slots <= p["max_slots"], (p, items, slots)
    return slots > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
def test_random_batches(dtype, d):
    rng = random.Random(d)
    size = lambda hi: int(round(hi ** rng.random()))
    cut = 0
    for _ in range(3000):
        hkv = rng.choice((1, 2, 3, 8, 16, 40, 300))
        hq = hkv * rng.choice((1, 2, 4, 7, 8, 64))
        n, top, most = size(200), size(1 << 22), size(3000)
        lens = [size(top) for _ in range(n)]
        new = [rng.choice((0, 1, 1, size(most), most)) for _ in range(n)]
        if rng.random() < 0.3:
            lens, new = [top] * n, [most] * n
        cut += bool(_holds(dtype, d, hq, hkv, lens, new, rng.choice((None, max(lens) * 2 + 1)), rng.choice((0, 5))))
    assert cut > 300


@pytest.mark.parametrize("hq,hkv,lens,new", [
    (8, 1, [400 << 20], [6560]),                    # 205 tiles over more than 2^28 keys: pages may repeat
    (8, 1, [500 << 20, 1], [8192, 1]), (64, 8, [1 << 20], [1 << 20]), (64, 1, [500 << 20] * 3, [20000] * 3), (1, 1, [500 << 20], [1]),
    (16, 16, [300 << 20] * 2, [70000, 3]),
])
@pytest.mark.parametrize("d", [128, 64])
def test_very_long_caches(d, hq, hkv, lens, new):
    for dtype in ("bf16", "f32"):
        _holds(dtype, d, hq, hkv, lens, new)
