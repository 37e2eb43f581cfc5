"""Wide tiles at the edges: every kernel of tests/paged_shapes.py over layouts, infinities and NaN in places that rows see or do not see,
scores of all sizes, rows without keys, arrays that hold numbers out of bounds, rows that repeat and rows far apart, captured steps."""
from functools import lru_cache

import numpy as np
import pytest

from tests import paged_bounds as B
from tests.paged_cases import Paged, check, rows_view
from tests.paged_shapes import PAGES, PROMPTS
from tests.test_gpu_prefill_attention import _case, _run

pytestmark = pytest.mark.gpu

WIDE_PAGES = [n for n in PAGES if not n.startswith(("few", "token"))]
WIDE_PROMPTS = [n for n in PROMPTS if not n.startswith("few")]


def _pages(name, extra=0):
    _, _, _, d, hq, hkv, page, lens, new = PAGES[name]
    return Paged(sum(lens) + d, "bf16", d, hq, hkv, page, lens, new, extra_rows=extra)


def _attend(x, layout="heads"):
    """Outputs on the host, and whether partial results were written (the workspace starts as 0xFF)."""
    import torch
    from paper_2508_11661_amd import samkv as S
    cache, batch = x.handles(S)
    out, lse = x.outputs(layout)
    ws = torch.full((S.samkv_paged_workspace_bytes(cache, batch, x.hq),), 0xFF, dtype=torch.uint8, device="cuda")
    S.samkv_paged_attn(cache, batch, rows_view(x.q, x.dtype, layout), x.scale, out, lse, ws)
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), bool((ws != 0xFF).any())


def _hold(out, lse, ref, d, scale, what):
    check(out, lse, ref, d, scale, "bf16", what)
    worst = B.two_term_error(out, ref, d, scale)
    assert worst <= 1.0, f"{what}: error {worst:.3g} of the bound of two-term weights"
    assert (out[:, ~ref.written] == 7.0).all() and (lse[:, ~ref.written] == 7.0).all(), f"{what}: rows of no sequence were written"


@lru_cache(maxsize=1)
def _pages_and_reference(name):
    x = _pages(name, extra=3)
    return x, B.pages(x)


@pytest.mark.parametrize("name", PAGES)
@pytest.mark.parametrize("layout", ["heads", "tokens", "part"])
def test_pages(name, layout):
    x, ref = _pages_and_reference(name)
    out, lse, parts = _attend(x, layout)
    _hold(out, lse, ref, x.d, x.scale, name)
    assert parts == PAGES[name][2], "keys cut, or not"


@lru_cache(maxsize=1)
def _prompts_and_reference(name):
    _, d, hq, hkv, lens = PROMPTS[name]
    (q, k, v), cu = _case(sum(lens) + d, "bf16", d, hq, hkv, lens, extra=3)
    return q, k, v, cu, B.prompts(q, k, v, cu, d ** -0.5)


@pytest.mark.parametrize("name", PROMPTS)
@pytest.mark.parametrize("layout", ["heads", "tokens", "part"])
def test_prompts(name, layout):
    q, k, v, cu, ref = _prompts_and_reference(name)
    d = q.shape[2]
    out, lse = _run("bf16", q, k, v, cu, int(np.diff(cu).max()), d ** -0.5, layout)
    _hold(out, lse, ref, d, d ** -0.5, name)


@pytest.mark.parametrize("name", [n for n in WIDE_PAGES if "empty" not in n])
def test_later_tokens_do_not_reach_a_row_of_pages(name):
    x = _pages(name)
    clean, clean_lse, _ = _attend(x)
    n, m = x.new[0], x.lens[0]
    at = lambda slot: (x.table[0, slot // x.page], slice(None), slot % x.page)
    for slot, value, ch in [(m - 2, np.nan, 3), (m - n // 2, np.inf, x.d - 1), (m - n + 1, -np.inf, 0)]:
        x.v[(*at(slot), ch)] = value
    out, lse, _ = _attend(x)
    ref = B.pages(x)
    assert (~np.isfinite(ref.out)).any()
    _hold(out, lse, ref, x.d, x.scale, f"{name}, values")
    x = _pages(name)
    x.k[(*at(m - n // 2), 5)] = np.nan
    out, lse, _ = _attend(x)
    same = np.r_[0:n - n // 2, n:x.n_rows]
    assert np.array_equal(out[:, same], clean[:, same]) and np.array_equal(lse[:, same], clean_lse[:, same])
    assert np.isnan(out[:, n - n // 2:n]).all() and np.isnan(lse[:, n - n // 2:n]).all()


@pytest.mark.parametrize("name", WIDE_PROMPTS)
def test_later_rows_do_not_reach_a_row_of_prompts(name):
    _, d, hq, hkv, lens = PROMPTS[name]
    (q, k, v), cu = _case(sum(lens) + d, "bf16", d, hq, hkv, lens)
    scale, n = d ** -0.5, lens[0]
    clean, clean_lse = _run("bf16", q, k, v, cu, max(lens), scale)
    v2, k2 = v.copy(), k.copy()
    for at, value, ch in [(n - 2, np.nan, 3), (n // 2, np.inf, d - 1), (1, -np.inf, 0), (sum(lens) - 1, np.nan, 1)]:
        v2[:, at, ch] = value
    out, lse = _run("bf16", q, k, v2, cu, max(lens), scale)
    ref = B.prompts(q, k, v2, cu, scale)
    assert (~np.isfinite(ref.out)).any()
    _hold(out, lse, ref, d, scale, f"{name}, values")
    k2[:, n // 2, 7] = np.nan
    out, lse = _run("bf16", q, k2, v, cu, max(lens), scale)
    same = np.r_[0:n // 2, n:sum(lens)]
    assert np.array_equal(out[:, same], clean[:, same]) and np.array_equal(lse[:, same], clean_lse[:, same])
    assert np.isnan(out[:, n // 2:n]).all()


@pytest.mark.parametrize("name", ["wide_cut_d128", "wide_cut_d64", "wide_steps_d128", "mid_cut_d128", "mid_cut_d64", "mid_d128", "mid_d64"])
def test_scores_of_all_sizes_over_pages(name):
    """Running maxima that rise and fall by far more than 2^8, and rows whose weights all sit on one key."""
    x = _pages(name)
    ramp = np.float32(2.0) ** np.random.default_rng(3).integers(-6, 4, x.k.shape[:1] + x.k.shape[2:3]).astype(np.float32)
    x.k *= ramp[:, None, :, None]
    out, lse, _ = _attend(x)
    _hold(out, lse, B.pages(x), x.d, x.scale, name)


@pytest.mark.parametrize("name", WIDE_PROMPTS)
def test_scores_of_all_sizes_over_prompts(name):
    _, d, hq, hkv, lens = PROMPTS[name]
    (q, k, v), cu = _case(sum(lens) + d, "bf16", d, hq, hkv, lens)
    k *= np.float32(2.0) ** np.random.default_rng(4).integers(-6, 4, k.shape[:2])[..., None].astype(np.float32)
    out, lse = _run("bf16", q, k, v, cu, max(lens), d ** -0.5)
    _hold(out, lse, B.prompts(q, k, v, cu, d ** -0.5), d, d ** -0.5, name)


@pytest.mark.parametrize("name,max_len,max_new", [("wide_d128", 120, 90), ("wide_d64", 120, 90), ("mid_d128", 300, 340), ("mid_d64", 300, 340)])
def test_values_beyond_bounds_stay_inside(name, max_len, max_new):
    """Lengths above max_len and below zero, prefix sums that run past the rows or backwards, more new tokens than max_new."""
    from tests import paged_plan
    x = _pages(name, extra=2)
    x.max_len, x.max_new = max_len, max_new
    x.lens[0], x.lens[1], x.lens[2] = 1000000, -5, 20
    x.cu = x.cu.copy()
    x.cu[0], x.cu[-1] = -3, 1 << 30
    p = paged_plan.plan("bf16", x.d, x.hq, x.hkv, len(x.lens), x.n_rows, max_new, max_len, True)
    assert p["kg"] == PAGES[name][0]
    out, lse, _ = _attend(x)
    _hold(out, lse, B.pages(x), x.d, x.scale, name)
    x.cu[0] = x.cu[1] + 7                            # backwards: no rows
    out, lse, _ = _attend(x)
    _hold(out, lse, B.pages(x), x.d, x.scale, name)


@pytest.mark.parametrize("name", ["wide_even_d128", "wide_even_d64", "mid_two_d128", "mid_two_d64"])
def test_prompts_longer_than_their_bound(name):
    from tests import paged_plan
    kg, d, hq, hkv, lens = PROMPTS[name]
    (q, k, v), cu = _case(sum(lens) + d, "bf16", d, hq, hkv, lens)
    most = max(lens) - 20
    assert paged_plan.plan("bf16", d, hq, hkv, len(lens), sum(lens), most, most, False)["kg"] == kg
    bound = np.stack([cu[:-1], np.minimum(cu[1:], cu[:-1] + most)])
    ref = B.P.Attention(hq, sum(lens), d)
    for a, b in bound.T:
        for h in range(hq):
            g = h * hkv // hq
            ref.put(h, a, b - a, b - a, B.attend_rows(q[h, a:b], k[g, a:b], v[g, a:b], d ** -0.5))
    out, lse = _run("bf16", q, k, v, np.r_[cu[:-1], 1 << 30], most, d ** -0.5)
    _hold(out, lse, ref, d, d ** -0.5, name)


def _prefill(q, k, v, lens, out):
    import torch
    from paper_2508_11661_amd import samkv as S
    n = sum(lens)
    cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    lse = torch.empty((q.shape[0], n), device="cuda")
    S.samkv_prefill_attn(q, k, v, cu, max(lens), q.shape[2] ** -0.5, out, lse, None)
    return out, lse


@pytest.mark.parametrize("name", WIDE_PROMPTS)
def test_rows_that_repeat(name):
    import torch
    _, d, hq, hkv, lens = PROMPTS[name]
    n = sum(lens)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for heads, rows in [(False, True), (True, False), (True, True)]:  # one head for all, one row for all
        sized = lambda h: torch.randn((1 if heads else h, 1 if rows else n, d), device="cuda", generator=gen).to(torch.bfloat16).expand(h, n, d)
        q, k, v = sized(hq), sized(hkv), sized(hkv)
        a = _prefill(q, k, v, lens, torch.empty((hq, n, d), dtype=q.dtype, device="cuda"))
        b = _prefill(*(x.contiguous() for x in (q, k, v)), lens, torch.empty((hq, n, d), dtype=q.dtype, device="cuda"))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def _far(x, head, row):
    """x at other strides, its elements that far apart."""
    import torch
    h, n, d = x.shape
    y = torch.empty(((h - 1) * head + (n - 1) * row + d,), dtype=x.dtype, device="cuda").as_strided((h, n, d), (head, row, 1))
    return y.copy_(x)


@pytest.mark.parametrize("name,head,row", [
    ("wide_uneven_d128", 5 << 27, 256), ("wide_uneven_d64", 5 << 27, 64), ("mid_one_d128", 5 << 28, 128), ("mid_one_d64", 5 << 28, 80),
    ("wide_uneven_d128", 128, (1 << 23) - 8), ("wide_uneven_d64", 64, (1 << 23) - 8),   # rows 16 MB less 16 bytes
    ("mid_one_d128", 128, (1 << 23) - 8), ("mid_one_d64", 72, (1 << 23) - 8),
])
def test_rows_beyond_32_bits(name, head, row):
    """Keys and values of up to 40 GB, queries and outputs of more than 4 GB: the bits of the same values in dense tensors."""
    import torch
    _, d, hq, hkv, lens = PROMPTS[name]
    n = sum(lens)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((h, n, d), device="cuda", generator=gen).to(torch.bfloat16) for h in (hq, hkv, hkv))
    want = _prefill(q, k, v, lens, torch.empty_like(q))
    wide = ((5 << 30) // hq // 16 * 16, d)
    got = _prefill(_far(q, *wide), _far(k, head, row), _far(v, head, row), lens, _far(torch.zeros_like(q), *wide))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name", ["few_d128", "wide_d128", "wide_cut_d64", "mid_d64", "mid_cut_d128", "token_d64"])
def test_queries_and_outputs_over_pages_repeat_or_lie_far_apart(name):
    import torch
    from paper_2508_11661_amd import samkv as S
    x = _pages(name)
    cache, batch = x.handles(S)
    ws = torch.empty((S.samkv_paged_workspace_bytes(cache, batch, x.hq),), dtype=torch.uint8, device="cuda")

    def run(q, out):
        lse = torch.empty((x.hq, x.n_rows), device="cuda")
        S.samkv_paged_attn(cache, batch, q, x.scale, out, lse, ws)
        return out, lse

    q = rows_view(x.q, "bf16", "heads")
    row = (5 << 30) // max(x.n_rows - 1, 1) // 16 * 16
    for this in (q[:1].expand_as(q), q[:, :1].expand_as(q), q[:1, :1].expand_as(q), _far(q, (5 << 30) // x.hq // 16 * 16, x.d), _far(q, x.d, row)):
        want = run(this.contiguous(), torch.empty_like(q))
        far = this.stride(0) * this.shape[0] > 1 << 31 or this.stride(1) * this.shape[1] > 1 << 31
        got = run(this, _far(torch.zeros_like(q), *this.stride()[:2]) if far else torch.empty_like(q))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_appended_rows_repeat_or_lie_far_apart(dtype):
    import torch
    from paper_2508_11661_amd import samkv as S
    x = Paged(5, dtype, 128, 6, 2, 16, [70, 300, 9], [33, 120, 9])
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v, q = (torch.randn((h, x.n_rows, x.d), device="cuda", generator=gen).to(rows_view(x.q, dtype, "heads").dtype) for h in (2, 2, 6))
    rope = S.Rope((10000.0 ** (-torch.arange(64, device="cuda") / 64.0)).float())

    def run(k, v, q, q_out):
        cache, batch = x.handles(S)
        cache.k.zero_(), cache.v.zero_()
        S.samkv_paged_append(cache, batch, k, v, rope, q, q_out)
        return cache.k, cache.v, q_out

    for view in (lambda t: t[:1].expand_as(t), lambda t: t[:, :1].expand_as(t), lambda t: _far(t, 1 << 31, x.d), lambda t: _far(t, x.d, 1 << 24)):
        parts = [view(t) for t in (k, v, q)]
        want = run(*(t.contiguous() for t in parts), torch.empty_like(q))
        far = min(parts[2].stride()[:2]) > 0
        got = run(*parts, view(torch.zeros_like(q)) if far else torch.empty_like(q))
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("new,kg", [([400, 500, 300, 402], 1), ([200, 230, 100, 270], 2)])
@pytest.mark.parametrize("d", [128, 64])
def test_a_captured_step_follows_the_batch(d, new, kg):
    """Append and attention of chunks in one graph; between replays the lengths, the table's rows, the tokens and the split of the rows
    over the sequences change on the device, with eager work in between.  Every replay gives the bits of the eager calls."""
    import torch
    from paper_2508_11661_amd import samkv as S
    from tests import paged_plan
    hq, hkv, page, n_pages, room = 32, 8, 16, 4 * 375, 6000
    gen = torch.Generator(device="cuda").manual_seed(3)
    R = lambda *s: torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16)
    I = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    n = sum(new)
    p = paged_plan.plan("bf16", d, hq, hkv, 4, n, max(new), room, True)
    assert p["kg"] == kg and p["joins"] == 1
    k_pages, v_pages = R(n_pages, hkv, page, d), R(n_pages, hkv, page, d)
    cache, eager = S.PagedCache(k_pages, v_pages), S.PagedCache(k_pages.clone(), v_pages.clone())
    table = torch.randperm(n_pages, device="cuda", generator=gen).view(4, 375).to(torch.int32).contiguous()
    lens, cu = I([600, 550, 5400, 440]), I(np.concatenate([[0], np.cumsum(new)]).tolist())
    batch = S.PagedBatch(table, lens, room, cu, max(new), n)
    rope = S.Rope((10000.0 ** (-torch.arange(d // 2, device="cuda") * 2.0 / d)).float())
    q, k, v = R(hq, n, d), R(hkv, n, d), R(hkv, n, d)
    ws = torch.full((S.samkv_paged_workspace_bytes(cache, batch, hq),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(cache, q_rot, out, lse):
        S.samkv_paged_append(cache, batch, k, v, rope, q, q_rot)
        S.samkv_paged_attn(cache, batch, q_rot, d ** -0.5, out, lse, ws)

    mine = [torch.zeros_like(q), torch.zeros_like(q), torch.zeros((hq, n), device="cuda")]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run(cache, *mine)
        run(eager, *mine)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(cache, *mine)
    for turn in range(4):
        lens.add_(I([1, 7, 60, 0]))
        if turn == 2:
            table.copy_(table.flip(0).clone())
        if turn == 3:
            cu.copy_(I([0, 0, max(new), max(new) + 1, n - 5]))
        for x in (q, k, v):
            x.copy_(R(*x.shape))
        for x in mine:
            x.fill_(7.0)
        graph.replay()
        theirs = [torch.full_like(x, 7.0) for x in mine]
        run(eager, *theirs)
        torch.cuda.synchronize()
        for a, b in zip(mine + [cache.k, cache.v], theirs + [eager.k, eager.v]):
            assert torch.equal(a, b), turn


def test_graphs_of_wide_tiles_share_a_workspace_and_streams_do_not():
    import torch
    from paper_2508_11661_amd import samkv as S
    sides = []
    for name in ("wide_cut_d128", "mid_cut_d64", "few_d128"):
        p = _pages(name)
        cache, batch = p.handles(S)
        out, lse = p.outputs()
        sides.append((p, cache, batch, rows_view(p.q, "bf16", "heads"), out, lse, S.samkv_paged_workspace_bytes(cache, batch, p.hq)))
    fresh = lambda n: torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    shared = fresh(max(s[-1] for s in sides))
    call = lambda s, ws: S.samkv_paged_attn(s[1], s[2], s[3], s[0].scale, s[4], s[5], ws)
    want = []
    for s in sides:
        call(s, fresh(s[-1]))
        want.append((s[4].clone(), s[5].clone()))
    graphs = []
    for s in sides:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(s, shared)
        graphs.append(g)
    for _ in range(3):
        for s, g, w in zip(sides, graphs, want):
            s[4].fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(s[4], w[0]) and torch.equal(s[5], w[1])
    streams, own = [torch.cuda.Stream() for _ in sides], [fresh(s[-1]) for s in sides]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, stream, ws in zip(sides, streams, own):
            with torch.cuda.stream(stream):
                call(s, ws)
    torch.cuda.synchronize()
    for s, w in zip(sides, want):
        assert torch.equal(s[4], w[0]) and torch.equal(s[5], w[1])
