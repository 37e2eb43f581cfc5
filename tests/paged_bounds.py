"""Float64 references on the device and element-wise bounds for attention over packed prompts and pages at sizes that the numpy
oracle is too slow for."""
from __future__ import annotations

import numpy as np

from oracle import paged_oracle as P

U = 2.0 ** -24


def attend_rows(q, k, v, scale, device="cuda"):
    """P.attend_rows in float64 on a device, at most 4096 rows at a time: q [n, d] are the newest rows of the keys k, v [m, d]."""
    import torch
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device).double()
    q, k, v = dev(q), dev(k), dev(v)
    n, m = len(q), len(k)
    if m == 0:
        return np.zeros(q.shape), np.full(n, -np.inf), np.zeros(q.shape), np.zeros(n)
    bad = ~torch.isfinite(v)
    clean = torch.where(bad, 0.0, v)
    kinds = [x.double() for x in (torch.isnan(v), v == np.inf, v == -np.inf)]
    parts = []
    for a in range(0, n, 4096):
        b = min(n, a + 4096)
        seen = torch.arange(m, device=device)[None] <= torch.arange(m - n + a, m - n + b, device=device)[:, None]
        s = (scale * (q[a:b] @ k.T)).masked_fill(~seen, -np.inf)
        top = s.amax(1, keepdim=True)
        w = torch.exp(s - torch.where(top == -np.inf, 0.0, top))
        total = w.sum(1, keepdim=True)
        some = torch.where(total == 0, 1.0, total)
        out, mean_abs = w @ clean / some, w @ clean.abs() / some
        if bad.any():  # a value that is not finite reaches the rows that see it
            nan, up, down = (seen.double() @ x > 0 for x in kinds)
            out = torch.where(up, np.inf, torch.where(down, -np.inf, out))
            out = torch.where(nan | (up & down), np.nan, out)
            mean_abs = torch.where(up | down, np.inf, mean_abs)
            mean_abs = torch.where(nan, np.nan, mean_abs)
        if total.isnan().any():  # a score that is NaN
            out, mean_abs = (torch.where(total.isnan(), np.nan, x) for x in (out, mean_abs))
        size = (q[a:b].abs() @ k.abs().T).masked_fill(~seen, 0.0).amax(1)
        parts.append((out, (top + total.log())[:, 0], mean_abs, size))
    return tuple(torch.cat(x).cpu().numpy() for x in zip(*parts))


def prompts(q, k, v, cu, scale):
    hq, n_rows, d = q.shape
    r = P.Attention(hq, n_rows, d)
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(hq):
            g = h * len(k) // hq
            if b > a:
                r.put(h, a, b - a, b - a, attend_rows(q[h, a:b], k[g, a:b], v[g, a:b], scale))
    return r


def pages(x):
    """Of a tests.paged_cases.Paged."""
    r = P.Attention(x.hq, x.n_rows, x.d)
    for s, (first, n, m) in enumerate(P.spans(len(x.lens), x.n_rows, x.max_new, x.max_len, x.cu, x.lens)):
        for h in range(x.hq if n else 0):
            g = h * x.hkv // x.hq
            r.put(h, first, n, m, attend_rows(x.q[h, first:first + n], P.cached(x.k, x.table[s], m, g), P.cached(x.v, x.table[s], m, g),
                                              x.scale))
    return r


def two_term_error(got_out, ref, d, scale):
    """Largest error of bf16 outputs, in units of what softmax weights of two bf16 terms allow.

    A weight p becomes hi + lo: |p - hi| <= 2^-8 p and the rest is rounded by at most 2^-8 of itself, so 2^-16 p is lost.  Scores and
    exponentials as in paged_cases.check (e), sums of 2 n products 2 n u; all that relative to the weighted mean of |v|.  The output is
    rounded once, by at most half a step of its type: 2^-8 of its value."""
    n = np.maximum(ref.seen, 1)[None, :, None]
    e = ((d + 2) * U * scale * ref.size + 4 * U * (1 + scale * ref.size))[..., None]
    rel = 2 * e + (2 * n + 8) * U + 2.0 ** -16
    bound = rel * ref.mean_abs * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(ref.out) + 1e-30
    fine = np.isfinite(ref.out) & ref.written[None, :, None]
    with np.errstate(invalid="ignore"):
        return float((np.abs(got_out.astype(np.float64) - ref.out) / bound)[fine].max())
