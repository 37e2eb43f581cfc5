"""Rows that repeat (strides of zero) and rows far apart (offsets beyond 32 bits): the bits of the same values in dense tensors."""
import pytest

from tests import helpers as H

pytestmark = pytest.mark.gpu


def _prefill(S, torch, q, k, v, lens, out):
    n = sum(lens)
    cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    lse = torch.empty((q.shape[0], n), device="cuda")
    S.samkv_prefill_attn(q, k, v, cu, max(lens), q.shape[2] ** -0.5, out, lse, None)
    return out, lse


@pytest.mark.parametrize("dtype,d,lens", [("bf16", 128, [40, 7]), ("bf16", 128, [900, 3]), ("bf16", 64, [900, 3]), ("f32", 128, [90, 3])])
def test_rows_that_repeat(dtype, d, lens):
    import torch
    from paper_2508_11661_amd import samkv as S
    gen = torch.Generator(device="cuda").manual_seed(1)
    R = lambda *s: torch.randn(s, device="cuda", generator=gen).to(H.torch_dtype(dtype))
    hq, hkv, n = 8, 2, sum(lens)
    for shape in [(1, n, d), (-1, 1, d), (1, 1, d)]:
        sized = lambda heads: R(heads if shape[0] < 0 else 1, shape[1], d).expand(heads, n, d)
        q, k, v = sized(hq), sized(hkv), sized(hkv)
        a = _prefill(S, torch, q, k, v, lens, torch.empty((hq, n, d), dtype=q.dtype, device="cuda"))
        b = _prefill(S, torch, *(x.contiguous() for x in (q, k, v)), lens, torch.empty((hq, n, d), dtype=q.dtype, device="cuda"))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("d,lens,head,row", [
    (128, [700, 30], 5 << 28, 256), (64, [700, 30], 5 << 28, 64), (128, [20, 3], 5 << 28, 128),   # heads 2.5 GB apart
    (128, [260, 9], 128, (1 << 23) - 8), (64, [260, 9], 64, (1 << 23) - 8), (128, [20, 3], 128, (1 << 23) - 8),  # rows 16 MB less 16 bytes
])
def test_rows_beyond_32_bits(d, lens, head, row):
    import torch
    from paper_2508_11661_amd import samkv as S
    gen = torch.Generator(device="cuda").manual_seed(2)
    hq, hkv, n = 4, 2, sum(lens)

    def far(x):
        h = x.shape[0]
        y = torch.empty(((h - 1) * head + (n - 1) * row + d,), dtype=x.dtype, device="cuda").as_strided((h, n, d), (head, row, 1))
        return y.copy_(x)

    q, k, v = (torch.randn((h, n, d), device="cuda", generator=gen).to(torch.bfloat16) for h in (hq, hkv, hkv))
    want = _prefill(S, torch, q, k, v, lens, torch.empty_like(q))
    got = _prefill(S, torch, far(q), far(k), far(v), lens, far(torch.zeros_like(q)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
