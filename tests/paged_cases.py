"""Inputs, bounds and comparisons shared by the tests of the packed prefill and the paged cache."""
from __future__ import annotations

import math

import numpy as np

from oracle import paged_oracle as P
from paper_2508_11661_amd import synth


def draw(rng, shape, dtype, spread=1.5):
    return synth.round_to_dtype(rng.standard_normal(shape, dtype=np.float32) * spread, dtype)


def check(got_out, got_lse, ref, d, scale, dtype, what=""):
    """Outputs against the oracle's, element by element.  With A the weighted mean of |v| and u = 2^-24:
    a score, a float32 sum of d exact products (float32: rounded ones), is off by e <= (d + 2) u scale sum |q_c k_c|, the products
    with scale and log2(e) and the exponential by 4 u more, relative to the weight and to the score; a weight is off by twice that
    beside its rounding (numerator and denominator), and the sums over n keys by n u.  bf16: a weight is rounded by at most half
    a step, 2^-8 relative, and so is the output."""
    u = 2.0 ** -24
    w = ref.written
    fine = np.isfinite(ref.out) & w[None, :, None]  # values that rows see and that are not finite: the same in both
    other = ~fine & w[None, :, None]
    assert np.isfinite(got_out[fine]).all(), f"{what}: non-finite output"
    assert np.array_equal(got_out[other], ref.out[other], equal_nan=True), f"{what}: infinities and NaN"
    n = np.maximum(ref.seen, 1)[None]
    lse = np.where(np.isfinite(ref.lse), ref.lse, 0.0)
    e = (d + 2) * u * scale * ref.size + 4 * u * (1 + scale * ref.size)
    rel = 2 * e + (n + 8) * u + (2.0 ** -8 if dtype == "bf16" else 0.0)
    bound = rel[..., None] * ref.mean_abs * (1 + 2.0 ** -7) + (2.0 ** -8 * np.abs(ref.out) if dtype == "bf16" else 0.0) + 1e-30
    with np.errstate(invalid="ignore"):
        err = np.abs(got_out.astype(np.float64) - ref.out)
        worst = (err / bound)[fine].max() if fine.any() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3g} of its bound"
    if got_lse is not None:
        empty = ~np.isfinite(ref.lse) & w[None]
        assert np.all(np.isneginf(got_lse[empty])), f"{what}: log-sum-exp of rows without keys"
        full = np.isfinite(ref.lse) & w[None]
        bound = e + (n + 8) * u + 2 * u * np.abs(lse)
        worst = (np.abs(got_lse - lse) / bound)[full].max() if full.any() else 0.0
        assert worst <= 1.0, f"{what}: log-sum-exp error {worst:.3g} of its bound"


def rows_view(a, dtype, layout, device="cuda"):
    """[heads, rows, d] device tensor of the values of `a` in one of the layouts that a caller may have."""
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    t = torch.from_numpy(np.ascontiguousarray(a)).to(device).to(dt)
    h, n, d = t.shape
    if layout == "heads":
        return t.contiguous()
    if layout == "tokens":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((n + 3, h + 2, d + 16), float("nan"), dtype=dt, device=device)  # a part of a larger tensor
    view = wide[2:2 + n, 1:1 + h, 8:8 + d].transpose(0, 1)
    view.copy_(t)
    return view


class Paged:
    """A batch over pages in no order: unused slots, pages and table entries hold NaN and numbers out of range."""

    def __init__(self, seed, dtype, d, hq, hkv, page, lens, new, uniform=False, extra_rows=0, spare_pages=3, max_len=None):
        rng = np.random.default_rng(seed)
        self.dtype, self.d, self.hq, self.hkv, self.page = dtype, d, hq, hkv, page
        self.lens, self.new, self.scale = list(lens), list(new), 1.0 / math.sqrt(d)
        self.n_rows = sum(new) + extra_rows
        self.cu = None if uniform else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.max_new, self.max_len = max(max(new), 1), max(max(lens), 1) if max_len is None else max_len
        per = [-(-max(n, 0) // page) for n in lens]
        n_pages = sum(per) + spare_pages
        order = rng.permutation(n_pages)
        self.table = rng.choice(np.array([-1, -7, n_pages, 1 << 30]), (len(lens), max(1, -(-self.max_len // page)) + 2)).astype(np.int32)
        self.k = np.full((n_pages, hkv, page, d), np.nan, np.float32)
        self.v = np.full((n_pages, hkv, page, d), np.nan, np.float32)
        at = 0
        for s, n in enumerate(lens):
            mine = order[at:at + per[s]]
            self.table[s, :per[s]] = mine
            at += per[s]
            slots = np.arange(max(n, 0))
            for x in (self.k, self.v):
                x[mine[slots // page], :, slots % page] = draw(rng, (len(slots), hkv, d), dtype)
        self.q = draw(rng, (hq, self.n_rows, d), dtype)

    def oracle(self):
        return P.paged_attention(self.k, self.v, self.table, self.lens, self.max_len, self.q, self.scale, self.max_new, self.cu)

    def handles(self, S):
        import torch
        dt = {"f32": torch.float32, "bf16": torch.bfloat16}[self.dtype]
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
        cache = S.PagedCache(torch.from_numpy(self.k).cuda().to(dt), torch.from_numpy(self.v).cuda().to(dt))
        batch = S.PagedBatch(dev(self.table), dev(self.lens), self.max_len, None if self.cu is None else dev(self.cu),
                             self.max_new, self.n_rows)
        return cache, batch

    def outputs(self, layout="heads"):
        import torch
        out = rows_view(np.full((self.hq, self.n_rows, self.d), 7.0, np.float32), self.dtype, layout)
        return out, torch.full((self.hq, self.n_rows), 7.0, device="cuda")

    def attend(self, S, layout="heads", with_lse=True):
        """Runs samkv_paged_attn over a workspace of garbage; float64 outputs on the host."""
        import torch
        cache, batch = self.handles(S)
        out, lse = self.outputs(layout)
        ws = torch.full((S.samkv_paged_workspace_bytes(cache, batch, self.hq),), 0xFF, dtype=torch.uint8, device="cuda")
        S.samkv_paged_attn(cache, batch, rows_view(self.q, self.dtype, layout), self.scale, out, lse if with_lse else None, ws)
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def check(self, S, layout="heads"):
        ref = self.oracle()
        out, lse = self.attend(S, layout)
        check(out, lse, ref, self.d, self.scale, self.dtype, f"{self.dtype} d={self.d} {self.lens} {self.new}")
        w = ref.written
        assert (out[:, ~w] == 7.0).all() and (lse[:, ~w] == 7.0).all(), "rows of no sequence were written"
        return out, lse
