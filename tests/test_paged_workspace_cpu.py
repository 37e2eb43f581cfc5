"""A workspace that is enough for a batch is enough for every smaller one, so that a program allocates once for its largest."""
import random

import pytest

from tests import paged_plan
from tests.test_abi_cpu import S  # noqa: F401
from tests.test_paged_cpu import FAKE, _batch, _pages


def _bytes(S, dtype, d, hq, hkv, n_seq, n_new, max_new, max_len):  # noqa: F811
    pages = _pages(S, size=1024, hkv=hkv, d=d, dtype=int(dtype == "bf16"))
    batch = _batch(S, n_seq=n_seq, max_pages=1 << 15, max_len=max_len, max_new=max_new, n_new=n_new, cu=FAKE)
    return S._lib.samkv_paged_workspace_bytes(pages, batch, hq)


def test_fewer_sequences_may_be_cut_where_many_are_not(S):  # noqa: F811
    """32 heads over 8, single tokens over up to 2048 keys: 64 sequences are not cut, 4 are."""
    need = lambda n: paged_plan.plan("bf16", 128, 32, 8, n, n, 1, 2048, True)["bytes"]
    assert need(64) == 0 < need(4)
    assert _bytes(S, "bf16", 128, 32, 8, 64, 64, 1, 2048) >= need(4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
def test_enough_for_every_smaller_batch(S, dtype, d):  # noqa: F811
    rng = random.Random(d)
    size = lambda hi: int(round(hi ** rng.random()))
    for _ in range(300):
        hkv = rng.choice((1, 2, 3, 8, 16, 300))
        hq = hkv * rng.choice((1, 2, 4, 7, 8))
        n_seq, max_len = size(4096), size(1 << 20)
        n_new = min(n_seq * size(4096), (1 << 22) // hq)
        max_new = min(size(4096), n_new)
        enough = _bytes(S, dtype, d, hq, hkv, n_seq, n_new, max_new, max_len)
        for _ in range(60):
            n, rows, new, most = size(n_seq), size(n_new), size(max_new), size(max_len)
            need = paged_plan.plan(dtype, d, hq, hkv, n, rows, new, most, True)["bytes"]
            assert need <= enough, (hq, hkv, (n_seq, n_new, max_new, max_len), (n, rows, new, most))
            assert need <= _bytes(S, dtype, d, hq, hkv, n, rows, new, most) <= enough


def test_workspaces_stay_small(S):  # noqa: F811
    """Parts of at most two chunks' worth of rows per compute unit: 68 MB for wide tiles, 34 MB for tiles of 32 rows."""
    assert _bytes(S, "bf16", 128, 32, 8, 64, 64, 1, 8192) <= 4 << 20
    assert _bytes(S, "bf16", 128, 64, 8, 4096, 1 << 16, 4096, 1 << 20) <= 68 << 20
    assert _bytes(S, "f32", 128, 64, 8, 4096, 1 << 16, 4096, 1 << 20) <= 34 << 20
