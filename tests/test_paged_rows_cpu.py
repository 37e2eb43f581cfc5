"""How many rows a call may have: more than 2^23 queries (131072 tokens of 64 heads, say) are accepted, what the grids cannot hold is
not.  Nothing is launched: the calls that pass write their output in place of an input, which is the last check."""
import pytest

from tests.test_abi_cpu import S  # noqa: F401
from tests.test_paged_cpu import FAKE, _batch, _pages, _rows


@pytest.mark.parametrize("hq,hkv,n,code", [(64, 8, 1 << 17, -1), (64, 8, 1 << 20, -1), (8, 1, (1 << 24) - 1, -1), (8, 1, 1 << 24, -2), (64, 8, 1 << 21, -2)])
def test_rows(S, hq, hkv, n, code):  # noqa: F811
    ws, rows = FAKE * 256, lambda p, h: S._Rows(p, 128, 128 * h)
    assert S._lib.samkv_prefill_attn(rows(FAKE, hq), rows(FAKE * 2, hkv), rows(FAKE * 3, hkv), FAKE, 1024, n, 131072, hq, hkv, 128, 1, 0.1,
                                     rows(FAKE, hq), None, ws, 1 << 40, None) == code
    pages, batch = _pages(S, hkv=hkv, size=1024), _batch(S, n_seq=1024, max_pages=1024, max_len=1 << 20, max_new=131072, n_new=n, cu=FAKE)
    assert S._lib.samkv_paged_attn(pages, batch, rows(FAKE, hq), hq, 0.1, rows(FAKE, hq), None, ws, 1 << 40, None) == code
    assert (S._lib.samkv_paged_workspace_bytes(pages, batch, hq) > 0) == (code == -1)
    assert S._lib.samkv_paged_append(pages, batch, rows(FAKE * 2, hkv), rows(FAKE * 3, hkv), None, rows(FAKE, hq), rows(FAKE * 2, hq), hq,
                                     None) == code


@pytest.mark.parametrize("n,code", [((1 << 26) - 4, -1), ((1 << 26) - 3, -2)])
def test_tokens_of_an_append(S, n, code):  # noqa: F811
    """A workgroup of 256 threads per four tokens: at most 2^32 - 1 threads."""
    rows = lambda p: S._Rows(p, 128, 128)
    batch = _batch(S, n_seq=4096, max_pages=1024, max_len=16384, max_new=16384, n_new=n, cu=FAKE)
    assert S._lib.samkv_paged_append(_pages(S, hkv=1), batch, rows(FAKE * 2), rows(FAKE * 3), None, rows(FAKE), rows(FAKE * 2), 1, None) == code
