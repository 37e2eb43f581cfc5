"""Float64 references on the device and element-wise bounds for attention over packed prompts and pages at sizes that the numpy
oracle is too slow for."""
from __future__ import annotations

import numpy as np

from oracle import paged_oracle as P

U = 2.0 ** -24


def attend_rows(q, k, v, scale):
    """P.attend_rows in float64 on the device: q [n, d] are the newest rows of the keys k, v [m, d]; at most 4096 rows at a time."""
    import torch
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda().double()
    q, k, v = dev(q), dev(k), dev(v)
    n, m = len(q), len(k)
    parts = []
    for a in range(0, n, 4096):
        b = min(n, a + 4096)
        seen = torch.arange(m, device="cuda")[None] <= torch.arange(m - n + a, m - n + b, device="cuda")[:, None]
        s = (scale * (q[a:b] @ k.T)).masked_fill(~seen, -np.inf)
        top = s.amax(1, keepdim=True)
        w = torch.exp(s - top)
        total = w.sum(1, keepdim=True)
        size = (q[a:b].abs() @ k.abs().T).masked_fill(~seen, 0.0).amax(1)
        parts.append((w @ v / total, (top + total.log())[:, 0], w @ v.abs() / total, size))
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
    """Of a tests.paged_cases.Paged without rows that see nothing."""
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
    err = np.abs(got_out.astype(np.float64) - ref.out)
    return float((err / bound)[:, ref.written].max())
