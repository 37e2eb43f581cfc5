"""CPU-side checks of the packed prefill and the paged cache: the oracle against closed forms and brute force, and every refusal
of the entry points before anything is launched."""
import ctypes
import math

import numpy as np
import pytest

from oracle import paged_oracle as P
from tests.test_abi_cpu import S  # noqa: F401  (fixture: the binding, built if it is not)


# ---- oracle -------------------------------------------------------------------------------------------------------
def test_rows_are_softmax_averages_by_brute_force():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 4)), rng.standard_normal((5, 4)), rng.standard_normal((5, 4))
    out, lse, mean_abs, size = P.attend_rows(q, k, v, 0.7)
    for t in range(3):
        w = [math.exp(0.7 * sum(q[t, c] * k[j, c] for c in range(4))) for j in range(3 + t)]
        for c in range(4):
            assert out[t, c] == pytest.approx(sum(x * v[j, c] for j, x in enumerate(w)) / sum(w), rel=1e-12)
            assert mean_abs[t, c] == pytest.approx(sum(x * abs(v[j, c]) for j, x in enumerate(w)) / sum(w), rel=1e-12)
        assert lse[t] == pytest.approx(math.log(sum(w)), rel=1e-12)
        assert size[t] == pytest.approx(max(sum(abs(q[t, c] * k[j, c]) for c in range(4)) for j in range(3 + t)), rel=1e-12)


def test_rows_without_keys_and_with_one():
    q, k, v = np.ones((3, 2)), np.array([[1.0, 2.0]]), np.array([[3.0, -4.0]])
    out, lse, _, _ = P.attend_rows(q, k, v, 1.0)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.array_equal(out[2], v[0]) and lse[2] == 3.0


def test_prompts_do_not_see_each_other_and_equal_their_paged_form():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((4, 12, 8)), rng.standard_normal((2, 12, 8)), rng.standard_normal((2, 12, 8))
    cu = [0, 5, 5, 12]
    r = P.prefill(q, k, v, cu, 7, 0.3)
    alone = P.prefill(q[:, 5:], k[:, 5:], v[:, 5:], [0, 7], 7, 0.3)
    assert np.array_equal(r.out[:, 5:], alone.out) and r.written.all()
    table = np.array([[3, 9], [9, 9], [0, 2]])
    pages = np.full((4, 2, 4, 8), np.nan)
    kp, vp, _ = P.append(pages, pages, table, [5, 0, 7], 8, k, v, 7, cu)
    b = P.paged_attention(kp, vp, [[3, 3], [9, 9], [0, 2]], [5, 0, 7], 8, q, 0.3, 7, cu)
    assert np.allclose(b.out[:, 5:], r.out[:, 5:], rtol=1e-14) and np.allclose(b.out[:, :4], r.out[:, :4], rtol=1e-14)
    assert np.isnan(kp).any(axis=(1, 3)).sum() == 16 - 4 - 7    # page 9 does not exist: the fifth token has no place


def test_rotation_keeps_lengths_and_relative_angles():
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((1, 16)), rng.standard_normal((1, 16))
    inv = 100.0 ** (-np.arange(6) / 6)
    for inter in (False, True):
        a, b = P.rotate(x, 1000003, inv, inter), P.rotate(y, 1000001, inv, inter)
        assert np.linalg.norm(a) == pytest.approx(np.linalg.norm(x)) and np.array_equal(a[:, 12:], x[:, 12:])
        assert float((a * b).sum()) == pytest.approx(float((P.rotate(x, 2, inv, inter) * y).sum()), abs=1e-8)
        assert np.array_equal(P.rotate(x, 0, inv, inter), x)
    unit = np.zeros((1, 4))
    unit[0, 0] = 1.0
    assert np.allclose(P.rotate(unit, 1, [math.pi / 2, 0.0], False), [[0, 0, 1, 0]], atol=1e-15)
    assert np.allclose(P.rotate(unit, 1, [math.pi / 2, 0.0], True), [[0, 1, 0, 0]], atol=1e-15)


def test_spans_follow_the_stated_bounds():
    assert P.spans(4, 10, 3, 50, [-3, 2, 1, 8, 1 << 30], [99, -5, 4, 7]) == [(0, 2, 50), (2, 0, 0), (1, 3, 4), (8, 2, 7)]
    assert P.spans(2, 6, 3, 50, None, [1, 2]) == [(0, 3, 1), (3, 3, 2)]


# ---- refusals -----------------------------------------------------------------------------------------------------
FAKE = 0x1000  # never dereferenced: every call below must fail before any launch


def _rows(S, p=FAKE, hs=128, rs=1024):
    return S._Rows(p, hs, rs)


def _pages(S, n_pages=8, size=16, hkv=2, d=128, dtype=1, k=FAKE, v=FAKE):
    return S._Pages(n_pages, size, hkv, d, dtype, k, v)


def _batch(S, n_seq=2, max_pages=4, max_len=64, max_new=3, n_new=6, table=FAKE, lens=FAKE, cu=None):
    return S._Batch(n_seq, max_pages, max_len, max_new, n_new, table, lens, cu)


BAD_ROWS = [(dict(p=None), -1), (dict(p=FAKE + 8), -1), (dict(hs=-128), -1), (dict(rs=-8), -1), (dict(hs=129), -1),
            (dict(rs=1028), -1), (dict(hs=1 << 60), -2), (dict(rs=1 << 60), -2)]
OVERLAPPING = [dict(hs=0), dict(rs=0), dict(hs=120), dict(hs=128, rs=256), dict(hs=256, rs=128)]
BAD_BATCH = [(dict(n_seq=0), -1), (dict(max_pages=0), -1), (dict(max_len=0), -1), (dict(max_new=0), -1), (dict(n_new=0), -1),
             (dict(table=None), -1), (dict(lens=None), -1), (dict(table=FAKE + 2), -1), (dict(lens=FAKE + 1), -1),
             (dict(cu=FAKE + 2), -1), (dict(max_len=65), -1), (dict(n_new=7), -1), (dict(n_seq=5000, n_new=15000), -2),
             (dict(n_new=1 << 24, cu=FAKE), -2), (dict(max_pages=1 << 27, max_len=1 << 30), -2)]
BAD_PAGES = [(dict(n_pages=0), -1), (dict(size=0), -1), (dict(size=8), -2), (dict(size=24), -2), (dict(size=2048), -2),
             (dict(hkv=0), -1), (dict(hkv=3), -1), (dict(d=96), -2), (dict(dtype=2), -2), (dict(k=None), -1), (dict(v=None), -1),
             (dict(k=FAKE + 4), -1), (dict(v=FAKE + 8), -1)]


def test_refusals_of_paged_attention(S):  # noqa: F811
    def call(pages={}, batch={}, q={}, out={}, scale=0.1, lse=FAKE, hq=8, ws=FAKE * 256, n=1 << 40, no=()):
        a = dict(pages=_pages(S, **pages), batch=_batch(S, **batch), q=_rows(S, **q), out=_rows(S, **out))
        a = {k: None if k in no else x for k, x in a.items()}
        return S._lib.samkv_paged_attn(a["pages"], a["batch"], a["q"], hq, scale, a["out"], lse, ws, n, None)
    for name in ("pages", "batch", "q", "out"):
        assert call(no=(name,)) == -1, name
    for kw, code in BAD_ROWS:
        assert call(q=kw) == code and call(out=kw) == code, kw
    for kw in OVERLAPPING:
        assert call(out=kw) == -1, kw
    for kw, code in BAD_BATCH:
        assert call(batch=kw) == code, kw
        assert S.samkv_paged_workspace_bytes(type("C", (), dict(c=_pages(S))), type("B", (), dict(c=_batch(S, **kw))), 8) == 0
    for kw, code in BAD_PAGES:
        assert call(pages=kw) == code, kw
    for bad in (0.0, -1.0, math.inf, math.nan):
        assert call(scale=bad) == -1
    assert call(lse=FAKE + 2) == -1 and call(hq=7) == -1 and call(hq=0) == -1
    long = dict(max_pages=1000, max_len=16000)
    assert S._lib.samkv_paged_workspace_bytes(_pages(S), _batch(S, **long), 8) > 1024
    assert call(batch=long, ws=None) == -3 and call(batch=long, n=16) == -3 and call(batch=long, ws=FAKE * 256 + 16) == -3


def test_refusals_of_prefill(S):  # noqa: F811
    def call(q={}, k={}, v={}, out={}, cu=FAKE, n_seq=2, n=6, max_len=4, hq=8, hkv=2, d=128, dtype=1, scale=0.1, lse=FAKE, no=()):
        a = dict(q=_rows(S, **q), k=_rows(S, **k), v=_rows(S, **v), out=_rows(S, **out))
        a = {k: None if k in no else x for k, x in a.items()}
        return S._lib.samkv_prefill_attn(a["q"], a["k"], a["v"], cu, n_seq, n, max_len, hq, hkv, d, dtype, scale, a["out"], lse,
                                         FAKE * 256, 1 << 40, None)
    for name in ("q", "k", "v", "out"):
        assert call(no=(name,)) == -1, name
    for kw, code in BAD_ROWS:
        assert call(q=kw) == code and call(k=kw) == code and call(v=kw) == code and call(out=kw) == code, kw
    for kw in OVERLAPPING:
        assert call(out=kw) == -1, kw
    for kw, code in [(dict(cu=None), -1), (dict(cu=FAKE + 2), -1), (dict(n_seq=0), -1), (dict(n=0), -1), (dict(max_len=0), -1),
                     (dict(hq=7), -1), (dict(hq=0), -1), (dict(hkv=0), -1), (dict(d=80), -2), (dict(dtype=5), -2),
                     (dict(scale=0.0), -1), (dict(scale=math.nan), -1), (dict(lse=FAKE + 1), -1), (dict(n_seq=5000), -2),
                     (dict(n=1 << 24), -2), (dict(k=dict(rs=1 << 27)), -2), (dict(v=dict(rs=1 << 27)), -2)]:
        assert call(**kw) == code, kw
    assert S._lib.samkv_prefill_workspace_bytes(0, 6, 4, 8, 2, 128, 1) == 0


def test_refusals_of_append(S):  # noqa: F811
    def call(pages={}, batch={}, k={}, v={}, q={}, q_out={}, rope={}, hq=8, no=()):
        a = dict(pages=_pages(S, **pages), batch=_batch(S, **batch), k=_rows(S, **{"hs": 128, "rs": 256, **k}),
                 v=_rows(S, **{"hs": 128, "rs": 256, **v}), q=_rows(S, **q), q_out=_rows(S, **q_out),
                 rope=S._Rope(*{"inv_freq": FAKE, "rot": 128, "inter": 0, "pos": None, **rope}.values()))
        a = {k: None if k in no else x for k, x in a.items()}
        return S._lib.samkv_paged_append(a["pages"], a["batch"], a["k"], a["v"], a["rope"], a["q"], a["q_out"], hq, None)
    for name in ("pages", "batch", "k", "v", "q", "q_out"):
        assert call(no=(name,)) == -1, name
    for kw, code in BAD_ROWS:
        assert call(q=kw) == code and call(q_out=kw) == code and call(k=kw) == code and call(v=kw) == code, kw
    for kw in OVERLAPPING:
        assert call(q_out=kw) == -1, kw
    for kw, code in BAD_BATCH:
        assert call(batch=kw) == code, kw
    for kw, code in BAD_PAGES:
        assert call(pages=kw) == code, kw
    for kw, code in [(dict(inv_freq=None), -1), (dict(inv_freq=FAKE + 2), -1), (dict(pos=FAKE + 2), -1), (dict(rot=0), -1),
                     (dict(rot=144), -1), (dict(rot=31), -1), (dict(rot=24), -2)]:
        assert call(rope=kw) == code, kw
    assert call(hq=7) == -1


def test_handles_refuse_tensors_of_the_host(S):  # noqa: F811
    import torch
    with pytest.raises(AssertionError):
        S.PagedCache(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64))
    with pytest.raises(AssertionError):
        S.PagedBatch(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 8)
    with pytest.raises(AssertionError):
        S.Rope(torch.zeros(8))
