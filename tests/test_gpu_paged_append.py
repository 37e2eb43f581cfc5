"""Keys and values of new tokens into pages, with the rotation, against the float64 oracle: every page, rotated or left as it
was, and the queries beside them."""
import numpy as np
import pytest

from oracle import paged_oracle as P
from tests.paged_cases import Paged, draw, rows_view

pytestmark = pytest.mark.gpu


def _near(got, want, before, dtype, turned, what):
    """Rotated values: cos and sin are off by at most 2^-22 (the float32 rounding of the angle's half turn, 2^-25 of a turn, times 2 pi,
    and an ulp of the function), products and their sum by 2^-23, of a pair no longer than sqrt(2) times its larger value; then
    half a step of the type.  Everything else is a copy."""
    same = ~turned
    assert np.array_equal(got[same], want[same], equal_nan=True), f"{what}: copies"
    err = np.abs(got - want)[turned]
    bound = 2.0 ** -8 * np.abs(want[turned]) * (dtype == "bf16") + (2.0 ** -21 + 2.0 ** -22) * 1.5 * np.abs(before[turned])
    assert np.isfinite(got[turned]).all() and (err <= bound + 1e-30).all(), f"{what}: {np.max(err / (bound + 1e-30)):.3g} of the bound"


def _run(x, rot, interleaved, positions, base=10000.0, layout="heads", with_q=True, in_place=False):
    import torch
    from paper_2508_11661_amd import samkv as S
    rng = np.random.default_rng(99)
    k_new, v_new = draw(rng, (x.hkv, x.n_rows, x.d), x.dtype), draw(rng, (x.hkv, x.n_rows, x.d), x.dtype)
    inv = (base ** (-2.0 * np.arange(rot // 2) / max(rot, 1))).astype(np.float32)
    cache, batch = x.handles(S)
    rope = None
    if rot:
        pos = None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda()
        rope = S.Rope(torch.from_numpy(inv).cuda(), interleaved, pos)
    q = rows_view(x.q, x.dtype, layout)
    q_out = q if in_place else rows_view(np.full_like(x.q, 7.0), x.dtype, layout)
    S.samkv_paged_append(cache, batch, rows_view(k_new, x.dtype, layout), rows_view(v_new, x.dtype, layout), rope,
                         q if with_q else None, q_out if with_q else None)
    want_k, want_v, want_q = P.append(x.k, x.v, x.table, x.lens, x.max_len, k_new, v_new, x.max_new, x.cu,
                                      inv if rot else None, interleaved, positions, x.q if with_q else None,
                                      x.q if in_place else np.full_like(x.q, 7.0))
    # what a channel's pair holds before the rotation bounds its error
    size = lambda a: np.maximum(np.abs(a), np.roll(np.abs(a), 1, -1) + np.roll(np.abs(a), -1, -1) if interleaved else
                                np.concatenate([np.roll(np.abs(a[..., :rot]), rot // 2, -1), np.abs(a[..., rot:])], -1))
    old_k, old_v, _ = P.append(x.k, x.v, x.table, x.lens, x.max_len, size(k_new), v_new, x.max_new, x.cu)
    channel = np.broadcast_to(np.arange(x.d) < rot, x.k.shape)
    new = np.zeros(x.k.shape, bool)
    ones, _, _ = P.append(np.zeros_like(x.k), x.v, x.table, x.lens, x.max_len, np.ones_like(k_new), v_new, x.max_new, x.cu)
    new[:] = ones == 1.0
    host = lambda t: t.double().cpu().numpy()
    _near(host(cache.k), want_k, old_k, x.dtype, new & channel, "k pages")
    assert np.array_equal(host(cache.v), want_v, equal_nan=True), "v pages"
    if with_q:
        rows = np.zeros(x.n_rows, bool)
        for first, n, _ in P.spans(len(x.lens), x.n_rows, x.max_new, x.max_len, x.cu, x.lens):
            rows[first:first + n] = True
        turned = np.broadcast_to(rows[None, :, None] & (np.arange(x.d) < rot), x.q.shape)
        _near(host(q_out), want_q, size(x.q), x.dtype, turned, "queries")


@pytest.mark.parametrize("dtype,d,rot", [("bf16", 128, 128), ("bf16", 64, 64), ("f32", 128, 128), ("f32", 64, 64), ("bf16", 128, 64),
                                         ("f32", 64, 16), ("bf16", 64, 48), ("f32", 128, 112), ("bf16", 128, 16), ("bf16", 128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(dtype, d, rot, interleaved):
    _run(Paged(d + rot, dtype, d, 6, 2, 16, [40, 1, 17, 300], [3, 1, 17, 130], extra_rows=2), rot, interleaved, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["heads", "tokens", "part"])
def test_layouts(dtype, layout):
    x = Paged(3, dtype, 128, 5, 1, 64, [70, 64, 9], [6, 64, 9])
    _run(x, 128, False, None, layout=layout)
    _run(x, 128, False, None, layout=layout, in_place=True)
    _run(x, 64, True, None, layout=layout, with_q=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    """Angles of positions up to 2^31: float64 keeps them, float32 would be off by whole turns."""
    x = Paged(4, dtype, 64, 4, 2, 16, [50, 30], [20, 30])
    pos = np.random.default_rng(1).integers(0, 2 ** 31 - 1, x.n_rows)
    pos[:6] = [0, 1, 2 ** 20, 2 ** 31 - 1, -1, -(2 ** 31)]
    _run(x, 64, False, pos)
    _run(x, 64, True, pos, base=500000.0)


def test_tokens_without_a_slot_or_a_page():
    """More new tokens than tokens, empty sequences, lengths and prefix sums out of bounds, page numbers out of range under a new
    token: such tokens are not written, and nothing else changes."""
    for dtype in ("bf16", "f32"):
        _run(Paged(5, dtype, 64, 4, 2, 16, [3, 0, 40, 0, 2], [7, 4, 0, 0, 2]), 64, False, None)
        _run(Paged(6, dtype, 64, 4, 4, 16, [0, 5, 0], [1] * 3, uniform=True), 64, False, None)
        x = Paged(7, dtype, 128, 4, 2, 16, [60, 60, 60], [20, 20, 20])
        x.table[0, 3], x.table[1, 2], x.table[2, 3] = -1, len(x.k), 1 << 30
        _run(x, 128, False, None)
        x = Paged(8, dtype, 64, 4, 2, 16, [60, 60, 60], [4, 4, 4])
        x.max_len, x.max_new, x.lens = 50, 3, [1000000, -5, 20]
        _run(x, 32, False, None)


def test_many_sequences():
    rng = np.random.default_rng(9)
    lens = [int(x) for x in rng.integers(0, 60, 300)]
    _run(Paged(9, "bf16", 64, 4, 2, 16, lens, [int(min(n, x)) for n, x in zip(lens, rng.integers(0, 9, 300))], extra_rows=7), 64, False, None)
    _run(Paged(10, "f32", 64, 4, 2, 16, lens, [1] * 300, uniform=True), 64, False, None)


def test_many_tokens():
    """Workgroups that take all heads, one of them with fewer tokens than it holds."""
    _run(Paged(11, "bf16", 64, 27, 9, 64, [2100, 2003, 1], [2100, 2003, 1]), 64, False, None)
