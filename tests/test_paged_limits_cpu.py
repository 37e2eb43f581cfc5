"""Calls that the packed prefill and the paged attention refuse beyond those of a single bad argument: outputs in place of an input,
grids that are too large, and workspace sizes of such calls.  Nothing is launched."""
import pytest

from tests.test_paged_cpu import FAKE, S, _batch, _pages, _rows  # noqa: F401


def test_outputs_in_place_of_an_input_are_refused(S):  # noqa: F811
    ws = FAKE * 256
    for same in ("q", "k", "v"):
        at = dict(q=FAKE * 2, k=FAKE * 3, v=FAKE * 4)
        r = {n: _rows(S, p) for n, p in at.items()}
        assert S._lib.samkv_prefill_attn(r["q"], r["k"], r["v"], FAKE, 2, 6, 4, 8, 2, 128, 1, 0.1, _rows(S, at[same]), None, ws, 1 << 40,
                                         None) == -1, same
    assert S._lib.samkv_paged_attn(_pages(S), _batch(S), _rows(S), 8, 0.1, _rows(S), None, ws, 1 << 40, None) == -1


@pytest.mark.parametrize("heads,n,size", [(65535, 128, -2), (4096, 128, -1)])
def test_grids_beyond_32_bits_are_refused(S, heads, n, size):  # noqa: F811
    """65535 heads of 128 sequences that may have 128 rows each are 128 * 65535 workgroups of 512 threads (65535 less than 2^32 - 1) and
    one more per head where keys may be cut, as those of 16000 are.  4096 heads are fewer, and the next check, of out in place of
    q, answers."""
    pages, batch = _pages(S, hkv=heads), _batch(S, n_seq=n, max_new=n, n_new=n, cu=FAKE, max_pages=1000, max_len=16000)
    rows = _rows(S, hs=128, rs=128 * heads)
    assert S._lib.samkv_paged_attn(pages, batch, rows, heads, 0.1, rows, None, FAKE * 256, 1 << 50, None) == size
    assert (S._lib.samkv_paged_workspace_bytes(pages, batch, heads) > 0) == (size == -1)


def test_workspaces_do_not_grow_with_padding(S):  # noqa: F811
    """Sequences without rows take no part in the bounds: 4096 of them beside one new token need what one sequence needs."""
    one = S._lib.samkv_paged_workspace_bytes(_pages(S), _batch(S, n_seq=1, max_new=1, n_new=1, cu=FAKE, max_pages=1000, max_len=16000), 8)
    many = S._lib.samkv_paged_workspace_bytes(_pages(S), _batch(S, n_seq=4096, max_new=1, n_new=1, cu=FAKE, max_pages=1000, max_len=16000),
                                              8)
    assert 0 < many <= one
