"""Causal attention of packed prompts against the float64 oracle."""
import numpy as np
import pytest

from oracle import paged_oracle as P
from tests.paged_cases import check, draw, rows_view

pytestmark = pytest.mark.gpu


def _run(dtype, q, k, v, cu, max_len, scale, layout="heads"):
    import torch
    from paper_2508_11661_amd import samkv as S
    hq, n, d = q.shape
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    out = rows_view(np.full((hq, n, d), 7.0, np.float32), dtype, layout)
    lse = torch.full((hq, n), 7.0, device="cuda")
    need = S.samkv_prefill_workspace_bytes(len(cu) - 1, n, max_len, hq, k.shape[0], d, dt)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    S.samkv_prefill_attn(*(rows_view(x, dtype, layout) for x in (q, k, v)),
                         torch.tensor(np.asarray(cu), dtype=torch.int32, device="cuda"), max_len, scale, out, lse, ws)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def _case(seed, dtype, d, hq, hkv, lens, extra=0):
    rng = np.random.default_rng(seed)
    n = sum(lens) + extra
    return [draw(rng, (h, n, d), dtype) for h in (hq, hkv, hkv)], np.concatenate([[0], np.cumsum(lens)])


@pytest.mark.parametrize("dtype,d,hq,hkv,lens", [
    ("bf16", 128, 8, 2, [1, 2, 31, 32, 33, 63, 64, 65, 0, 130]), ("bf16", 64, 8, 2, [257, 1, 128, 127, 5]),
    ("bf16", 128, 4, 4, [700, 3]), ("bf16", 64, 7, 1, [300, 299]), ("bf16", 128, 6, 2, [512, 511]), ("bf16", 64, 3, 1, [900]),
    ("bf16", 128, 1, 1, [1]), ("bf16", 128, 32, 8, [200] * 5), ("bf16", 64, 24, 8, [65] * 7), ("bf16", 128, 16, 1, [260, 17]),
    ("f32", 128, 8, 2, [1, 2, 31, 32, 33, 63, 64, 65, 0, 130]), ("f32", 64, 8, 2, [257, 1, 128]), ("f32", 128, 3, 1, [300]),
    ("f32", 64, 4, 4, [500, 7]), ("f32", 128, 32, 8, [90] * 3), ("f32", 64, 16, 1, [129]),
])
@pytest.mark.parametrize("layout", ["heads", "tokens", "part"])
def test_packed_lengths(dtype, d, hq, hkv, lens, layout):
    (q, k, v), cu = _case(sum(lens) + d, dtype, d, hq, hkv, lens, extra=3)
    scale = d ** -0.5
    ref = P.prefill(q, k, v, cu, max(lens), scale)
    out, lse = _run(dtype, q, k, v, cu, max(lens), scale, layout)
    check(out, lse, ref, d, scale, dtype, f"prefill {dtype} d={d} {lens}")
    assert (out[:, ~ref.written] == 7.0).all() and (lse[:, ~ref.written] == 7.0).all()


@pytest.mark.parametrize("dtype,d,hq,hkv,n", [("bf16", 128, 4, 1, 2500), ("bf16", 64, 2, 1, 4100), ("f32", 128, 2, 1, 1300)])
def test_long_prompts(dtype, d, hq, hkv, n):
    """Every row of a long prompt in float64 on the GPU, by plain products."""
    import torch
    (q, k, v), cu = _case(n, dtype, d, hq, hkv, [n])
    scale = d ** -0.5
    out, lse = _run(dtype, q, k, v, cu, n, scale)
    r = P.Attention(hq, n, d)
    r.written[:], r.seen[:] = True, np.arange(1, n + 1)
    dev = lambda x: torch.from_numpy(x).cuda().double()
    mask = torch.triu(torch.ones((n, n), dtype=torch.bool, device="cuda"), 1)
    for h in range(hq):
        qd, kd, vd = dev(q[h]), dev(k[h * hkv // hq]), dev(v[h * hkv // hq])
        s = (qd @ kd.T * scale).masked_fill(mask, -np.inf)
        p = torch.softmax(s, 1)
        r.out[h], r.mean_abs[h] = (p @ vd).cpu().numpy(), (p @ vd.abs()).cpu().numpy()
        r.lse[h] = torch.logsumexp(s, 1).cpu().numpy()
        r.size[h] = (qd.abs() @ kd.abs().T).masked_fill(mask, 0.0).amax(1).cpu().numpy()
    check(out, lse, r, d, scale, dtype, f"prefill {dtype} {n}")


@pytest.mark.parametrize("dtype,d,hq,hkv,n", [("bf16", 128, 4, 1, 300), ("bf16", 64, 2, 2, 600), ("f32", 128, 4, 2, 130),
                                             ("bf16", 128, 2, 1, 40)])
def test_later_rows_do_not_reach_a_row(dtype, d, hq, hkv, n):
    lens = [n, 50, n]
    (q, k, v), cu = _case(n, dtype, d, hq, hkv, lens)
    scale = d ** -0.5
    clean, clean_lse = _run(dtype, q, k, v, cu, n, scale)
    v2 = v.copy()
    for at, value, ch in [(n - 2, np.nan, 3), (n // 2, np.inf, d - 1), (1, -np.inf, 0), (n + 49, np.nan, 1), (n + 50, np.inf, 2)]:
        v2[:, at, ch] = value
    out, lse = _run(dtype, q, k, v2, cu, n, scale)
    # Rows that meet such values may be computed by other sums than before (each within the bound of check(), so the two runs
    # are within twice that of each other): what is finite is held to the oracle, not to the bits of the clean run.
    ref = P.prefill(q, k, v2, cu, n, scale)
    assert (~np.isfinite(ref.out)).any()
    check(out, lse, ref, d, scale, dtype, "with infinities and NaN among the values")
    k2 = k.copy()
    k2[:, n // 2, 7] = np.nan
    out, lse = _run(dtype, q, k2, v, cu, n, scale)
    same = np.r_[0:n // 2, n:2 * n + 50]
    assert np.array_equal(out[:, same], clean[:, same]) and np.isnan(out[:, n // 2:n]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds(dtype):
    """A sequence longer than max_len keeps its rows past the bound as they were; prefix sums past the rows end there."""
    (q, k, v), _ = _case(3, dtype, 64, 4, 2, [200])
    cu = np.array([0, 90, 100, 500])
    ref = P.prefill(q, k, v, cu, 60, 0.125)
    assert ref.written.sum() == 60 + 10 + 60
    out, lse = _run(dtype, q, k, v, cu, 60, 0.125)
    check(out, lse, ref, 64, 0.125, dtype)
    assert (out[:, ~ref.written] == 7.0).all() and (lse[:, ~ref.written] == 7.0).all()


def test_many_sequences():
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 40, 200)]
    for dtype, d in (("bf16", 128), ("bf16", 64), ("f32", 64)):
        (q, k, v), cu = _case(6, dtype, d, 4, 2, lens)
        ref = P.prefill(q, k, v, cu, 40, 0.125)
        out, lse = _run(dtype, q, k, v, cu, 40, 0.125)
        check(out, lse, ref, d, 0.125, dtype)
