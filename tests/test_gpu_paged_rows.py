"""Calls of 2^23 query rows: 131072 tokens of 64 heads, as one prompt and as many, over prompts and over pages."""
import pytest

from oracle import paged_oracle as P
from tests import paged_bounds as B
from tests.paged_cases import check

pytestmark = pytest.mark.gpu
HQ, HKV, D, N = 64, 8, 64, 1 << 17


def _qkv():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, HQ + 2 * HKV, D), device="cuda", generator=gen, dtype=torch.bfloat16).transpose(0, 1)
    return x[:HQ], x[HQ:HQ + HKV], x[HQ + HKV:]


def _hold(out, lse, q, k, v, heads, first, n, at, rows):
    """Rows `at` .. `at` + rows - 1 of the sequence of n tokens that starts at row `first`."""
    host = lambda t: t.float().cpu().numpy()
    for h in heads:
        g, here = h * HKV // HQ, slice(first + at, first + at + rows)
        r = P.Attention(1, rows, D)
        keys = slice(first, first + at + rows)
        r.put(0, 0, rows, at + rows, B.attend_rows(host(q[h, here]), host(k[g, keys]), host(v[g, keys]), D ** -0.5))
        got = host(out[h:h + 1, here])
        check(got, host(lse[h:h + 1, here]), r, D, D ** -0.5, "bf16", f"head {h}, rows from {at}")
        assert B.two_term_error(got, r, D, D ** -0.5) <= 1.0


def test_prompts():
    import torch
    from paper_2508_11661_amd import samkv as S
    q, k, v = _qkv()
    out, lse = torch.empty((N, HQ, D), device="cuda", dtype=torch.bfloat16).transpose(0, 1), torch.empty((HQ, N), device="cuda")
    for n in (N, 128):
        cu = torch.arange(0, N + 1, n, device="cuda", dtype=torch.int32)
        out.fill_(7.0)
        S.samkv_prefill_attn(q, k, v, cu, n, D ** -0.5, out, lse, None)
        for first in sorted({0, N // 2 // n * n, N - n}):
            for at in sorted({0, n // 2, n - 32}):
                _hold(out, lse, q, k, v, (0, 37, HQ - 1), first, n, at, 32)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_pages():
    """Appended in one call and in two, then attended from in one."""
    import torch
    from paper_2508_11661_amd import samkv as S
    q, k, v = _qkv()
    page, n, n_seq = 128, 512, N // 512
    caches = [S.PagedCache(*(torch.zeros((N // page, HKV, page, D), device="cuda", dtype=torch.bfloat16) for _ in range(2))) for _ in range(2)]
    table = torch.randperm(N // page, device="cuda").to(torch.int32).view(n_seq, n // page).contiguous()
    full = torch.full((n_seq,), n, dtype=torch.int32, device="cuda")
    rope = S.Rope((10000.0 ** (-torch.arange(D // 2, device="cuda") * 2.0 / D)).float())
    q_rot = [torch.empty((N, HQ, D), device="cuda", dtype=torch.bfloat16).transpose(0, 1) for _ in range(2)]
    whole = S.PagedBatch(table, full, n, None, n)
    S.samkv_paged_append(caches[0], whole, k, v, rope, q, q_rot[0])
    for a in (0, n_seq // 2):
        rows = slice(a * n, (a + n_seq // 2) * n)
        half = S.PagedBatch(table[a:a + n_seq // 2].contiguous(), full[:n_seq // 2], n, None, n)
        S.samkv_paged_append(caches[1], half, k[:, rows], v[:, rows], rope, q[:, rows], q_rot[1][:, rows])
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v) and torch.equal(*q_rot)
    out, lse = torch.empty((N, HQ, D), device="cuda", dtype=torch.bfloat16).transpose(0, 1), torch.empty((HQ, N), device="cuda")
    ws = torch.empty((max(S.samkv_paged_workspace_bytes(caches[0], whole, HQ), 1),), dtype=torch.uint8, device="cuda")
    S.samkv_paged_attn(caches[0], whole, q_rot[0], D ** -0.5, out, lse, ws)
    k_rot = torch.empty((HKV, N, D), device="cuda", dtype=torch.bfloat16)
    for s in (0, n_seq // 2, n_seq - 1):
        k_rot[:, s * n:(s + 1) * n] = caches[0].k[table[s].long()].transpose(0, 1).reshape(HKV, n, D)
        for at in (0, n // 2, n - 32):
            _hold(out, lse, q_rot[0], k_rot, v, (0, 37, HQ - 1), s * n, n, at, 32)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
