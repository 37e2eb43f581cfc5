"""Refusals of the paged append where what is written lies on what is read.  Nothing is launched."""
import pytest

from tests.test_abi_cpu import S  # noqa: F401
from tests.test_paged_cpu import FAKE, _batch, _pages, _rows


def _append(S, q, q_out, hq=8, n_seq=2, k=FAKE * 4, v=FAKE * 5):  # noqa: F811
    rope = S._Rope(FAKE, 128, 0, None)
    kv = lambda p: S._Rows(p, 128, 256)
    batch = _batch(S, n_seq=n_seq, max_new=3 if n_seq > 1 else 1, n_new=3 * n_seq if n_seq > 1 else 1)
    return S._lib.samkv_paged_append(_pages(S), batch, kv(k), kv(v), rope, q, q_out, hq, None)


@pytest.mark.parametrize("strides", [(1024 * 6, 128), (256, 2048), (128, 1032), (136, 1088)])
def test_queries_in_place_need_the_same_strides(S, strides):  # noqa: F811
    """q [6 tokens][8 heads][128]: any other strides would write rows that other workgroups have yet to read."""
    assert _append(S, _rows(S), S._Rows(FAKE, *strides)) == -1
    assert _append(S, S._Rows(FAKE, *strides), _rows(S)) == -1
    assert _append(S, S._Rows(FAKE, 0, 1024), _rows(S)) == -1     # one head's rows for all


def test_queries_in_place_of_keys_or_values_are_refused(S):  # noqa: F811
    for at in (FAKE * 4, FAKE * 5):
        assert _append(S, _rows(S), _rows(S, at)) == -1


def test_strides_of_single_heads_and_rows_do_not_count(S):  # noqa: F811
    """One token: its row stride says nothing, and the call passes this check (and every other: it reaches the launch, which fails
    without a device)."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would be launched")
    assert _append(S, S._Rows(FAKE, 128, 1024), S._Rows(FAKE, 128, 4096), n_seq=1) not in (-1, -2, -3)
    assert _append(S, _rows(S), _rows(S)) not in (-1, -2, -3)
