"""Operators of a serving program around the sparse path: prompts packed into one batch are prefilled, their keys and
values are appended to a paged cache with the rotary position embedding applied on the way, and new tokens attend over
that cache.

Three operators:
  prefill   causal attention over packed prompts of different lengths (`samkv_prefill_attn`)
  append    K and V of new tokens into pages, K and the queries rotated (`samkv_paged_append`)
  attend    attention of the new tokens of a batch over its paged cache (`samkv_paged_attn`)

Queries, keys and values are views of one projection's output [tokens, Hq + 2 Hkv, d], as a model's attention block has
them; outputs go to [tokens, Hq, d].  Values follow `synth.make_layer`: channel scales log-uniform in [0.5, 4].
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _prefill(name, dtype, n_seq, max_len, hq, hkv, d, ragged):
    return dict(name=name, op="prefill", dtype=dtype, n_seq=n_seq, max_len=max_len, hq=hq, hkv=hkv, d=d, ragged=ragged)


def _paged(name, op, dtype, n_seq, max_len, new, max_new, hq, hkv, d, page, rot=0, interleaved=False, positions="slot"):
    c = dict(name=name, op=op, dtype=dtype, n_seq=n_seq, max_len=max_len, new=new, max_new=max_new, hq=hq, hkv=hkv, d=d,
             page=page)
    return c if op == "attend" else dict(c, rot=rot, interleaved=interleaved, positions=positions)


def listed():
    return [
        # four short documents of a toy layer in float32: launches and latency
        _prefill("prefill_tiny_f32", "f32", 4, 256, 8, 2, 64, False),
        # the ordinary layer of `llama3_8b_layer`: ten retrieved documents prefilled together
        _prefill("prefill_documents", "bf16", 10, 1024, 32, 8, 128, False),
        # ragged passages, a small model's head dimension, three query heads per KV head
        _prefill("prefill_ragged_d64", "bf16", 23, 2999, 24, 8, 64, True),
        # a quarter of the documents of the largest layer
        _prefill("prefill_large", "bf16", 16, 4096, 64, 8, 128, False),
        # one decoding step of a small batch: a row of K and V per head and sequence
        _paged("append_token", "append", "bf16", 16, 4096, "each", 1, 32, 8, 128, 16, rot=128),
        # the documents of the budget sweep written into pages after their prefill, every document from position 0
        _paged("append_documents", "append", "bf16", 40, 2048, "whole", 2048, 32, 8, 128, 64, rot=128),
        # float32, rotation of a part of the channels in neighbouring pairs, ragged chunks, positions given apart
        _paged("append_ragged_f32", "append", "f32", 19, 3000, "ragged", 700, 14, 2, 64, 32, rot=32, interleaved=True,
               positions="given"),
        # one token of a few conversations
        _paged("attend_token_few", "attend", "bf16", 4, 2048, "each", 1, 32, 8, 128, 16),
        # a full decoding batch of ragged conversations
        _paged("attend_token_batch", "attend", "bf16", 64, 8192, "each", 1, 64, 8, 128, 16),
        # one token over one very long context
        _paged("attend_token_long", "attend", "bf16", 1, 131072, "each", 1, 32, 8, 128, 64),
        # continuous batching: decoding tokens beside chunks of prompts that are being prefilled
        _paged("attend_mixed_chunks", "attend", "bf16", 24, 12000, "mixed", 1024, 32, 8, 128, 32),
        # a few drafted tokens checked at once, float32 cache, head dimension 64
        _paged("attend_draft_f32", "attend", "f32", 7, 3333, "ragged", 6, 16, 4, 64, 16),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    while True:
        op = rng.choice(("prefill", "append", "attend", "attend"))
        dtype, d = rng.choice(("bf16", "bf16", "bf16", "f32")), rng.choice((128, 128, 64))
        hkv = rng.choice((1, 2, 4, 8, 8, 8))
        hq = hkv * rng.choice((1, 3, 4, 4, 7, 8))
        n_seq = _log_uniform(rng, 1, 64)
        if op == "prefill":
            c = _prefill(None, dtype, n_seq, _log_uniform(rng, 16, 16384), hq, hkv, d, rng.random() < 0.7)
        else:
            new = rng.choice(("each", "each", "ragged", "mixed", "whole"))
            max_len = _log_uniform(rng, 16, 131072)
            max_new = 1 if new == "each" else max_len if new == "whole" else min(max_len, _log_uniform(rng, 2, 2048))
            rot = rng.choice((d, d, d // 2, 16))
            c = _paged(None, op, dtype, n_seq, max_len, new, max_new, hq, hkv, d, rng.choice((16, 16, 32, 64, 128)), rot,
                       rng.random() < 0.3, rng.choice(("slot", "slot", "given")))
        del c["name"]
        w = work(c)
        pool = n_seq * c["max_len"] * hkv * d * (2 if dtype == "bf16" else 4)
        # no more than the largest listed case, and float32 products run at a small part of the bf16 rate
        if pool <= 3 << 29 and w["bytes"] <= 2 << 30 and w["flops"] <= (4e12 if dtype == "bf16" else 2e11):
            return c


# ---- shapes --------------------------------------------------------------------------------------------------------
def _lens(c):
    """Tokens per sequence, the new ones included: all max_len, or spread over [max_len / 8, max_len]."""
    r = random.Random(c["n_seq"] * 1000003 + c["max_len"])
    if c["op"] == "prefill" and not c["ragged"] or c.get("new") == "whole" or c["n_seq"] == 1:
        return [c["max_len"]] * c["n_seq"]
    return [c["max_len"]] + [r.randint(max(1, c["max_len"] // 8), c["max_len"]) for _ in range(c["n_seq"] - 1)]


def _new(c):
    """New tokens per sequence."""
    lens = _lens(c)
    if c["op"] == "prefill" or c["new"] == "whole":
        return lens
    r = random.Random(c["n_seq"] * 7919 + c["max_new"])
    if c["new"] == "each":
        return [min(n, c["max_new"]) for n in lens]
    if c["new"] == "ragged":
        return [min(n, c["max_new"] if i == 0 else r.randint(1, c["max_new"])) for i, n in enumerate(lens)]
    return [min(n, c["max_new"] if i % 8 == 0 else 1) for i, n in enumerate(lens)]  # mixed


def work(case):
    e, d, hq, hkv = (2 if case["dtype"] == "bf16" else 4), case["d"], case["hq"], case["hkv"]
    lens, new = _lens(case), _new(case)
    n = sum(new)
    if case["op"] == "append":
        return {"bytes": 2 * (2 * hkv + hq) * n * d * e + 4 * n, "flops": 3 * (hq + hkv) * n * case["rot"]}
    keys = sum(lens)  # each key and value once; a query row and its output once
    pairs = sum(m * (L - m) + m * (m + 1) // 2 for L, m in zip(lens, new))
    return {"bytes": 2 * hkv * keys * d * e + hq * n * (2 * d * e + 4), "flops": 4 * hq * d * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------------
class _State:
    pass


def prepare(case, seed):
    dev, dt = "cuda", torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=dev).manual_seed(seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens, new = _lens(case), _new(case)
    n = sum(new)
    s = _State()
    s.case, s.scale, s.dt, s.lens, s.new = case, 1.0 / math.sqrt(d), dt, lens, new

    def scales():
        return torch.exp(torch.empty((hkv, 1, d), device=dev).uniform_(math.log(0.5), math.log(4.0), generator=gen))

    def prefix(x):
        return torch.tensor([0] + torch.tensor(x).cumsum(0).tolist(), dtype=torch.int32, device=dev)

    sk, sv = scales(), scales()
    qkv = torch.randn((n, hq + 2 * hkv, d), device=dev, generator=gen, dtype=dt)
    qkv[:, hq:hq + hkv].mul_(sk.view(1, hkv, d).to(dt))
    qkv[:, hq + hkv:].mul_(sv.view(1, hkv, d).to(dt))
    heads = qkv.transpose(0, 1)
    s.q, s.k, s.v = heads[:hq], heads[hq:hq + hkv], heads[hq + hkv:]
    s.cu = prefix(new)
    s.out = torch.empty((n, hq, d), device=dev, dtype=dt).transpose(0, 1)
    s.lse = torch.empty((hq, n), device=dev)
    if case["op"] != "prefill":
        page = case["page"]
        per = [-(-x // page) for x in lens]
        s.lens_dev = torch.tensor(lens, dtype=torch.int32, device=dev)
        order = torch.randperm(sum(per), device=dev, generator=gen).to(torch.int32)  # pages in no order
        # sequence s owns the pages order[at[s]] ..; columns past its last page repeat that one
        at = torch.tensor([0] + per[:-1], device=dev).cumsum(0)
        col = torch.minimum(torch.arange(max(per), device=dev)[None], torch.tensor(per, device=dev)[:, None] - 1)
        s.table = order[at[:, None] + col].contiguous()
        s.k_pages = torch.randn((sum(per), hkv, page, d), device=dev, generator=gen, dtype=dt).mul_(sk.to(dt))
        s.v_pages = torch.randn((sum(per), hkv, page, d), device=dev, generator=gen, dtype=dt).mul_(sv.to(dt))
    if case["op"] == "append":
        # frequencies of a rotary embedding of base 500000; given positions lie anywhere in a long context
        i = torch.arange(case["rot"] // 2, device=dev, dtype=torch.float64)
        s.inv_freq = (500000.0 ** (-2.0 * i / case["rot"])).float()
        s.pos = None
        if case["positions"] == "given":
            s.pos = torch.randint(0, 1 << 20, (n,), device=dev, generator=gen, dtype=torch.int32)
        s.q_out = torch.empty_like(s.out)
    if own:  # what a serving program sets up once: handles of the cache and of the batch's buffers, and a workspace
        from paper_2508_11661_amd import samkv
        if case["op"] == "prefill":
            need = samkv.samkv_prefill_workspace_bytes(case["n_seq"], n, max(lens), hq, hkv, d, dt)
        else:
            s.cache = samkv.PagedCache(s.k_pages, s.v_pages)
            s.batch = samkv.PagedBatch(s.table, s.lens_dev, max(lens), s.cu, max(new), n)
            need = samkv.samkv_paged_workspace_bytes(s.cache, s.batch, hq)
            if case["op"] == "append":
                s.rope = samkv.Rope(s.inv_freq, case["interleaved"], s.pos)
        s.ws = torch.empty((max(need, 1),), dtype=torch.uint8, device=dev)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(state):
    s, c = state, state.case
    if c["op"] == "prefill":
        if own:
            from paper_2508_11661_amd import samkv
            samkv.samkv_prefill_attn(s.q, s.k, s.v, s.cu, max(s.lens), s.scale, s.out, s.lse, s.ws)
        else:
            at = 0
            for n in s.lens:
                _plain_causal(s, s.q[:, at:at + n], s.k[:, at:at + n], s.v[:, at:at + n], at)
                at += n
        return {"out": s.out, "lse": s.lse}
    if c["op"] == "append":
        if own:
            from paper_2508_11661_amd import samkv
            samkv.samkv_paged_append(s.cache, s.batch, s.k, s.v, s.rope, s.q, s.q_out)
        else:
            _plain_append(s)
        return {"k_pages": s.k_pages, "v_pages": s.v_pages, "q": s.q_out}
    if own:
        from paper_2508_11661_amd import samkv
        samkv.samkv_paged_attn(s.cache, s.batch, s.q, s.scale, s.out, s.lse, s.ws)
    elif max(s.new) * sum(s.lens) * c["hq"] <= 1 << 28:
        _plain_padded(s)
    else:
        at = 0
        for i, n in enumerate(s.new):
            _plain_causal(s, s.q[:, at:at + n], _cached(s, s.k_pages, i), _cached(s, s.v_pages, i), at)
            at += n
    return {"out": s.out, "lse": s.lse}


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _cached(s, pages, i):
    """[Hkv, len, d] of sequence i."""
    c = s.case
    used = s.table[i, :-(-s.lens[i] // c["page"])].long()
    return pages[used].transpose(0, 1).reshape(c["hkv"], -1, c["d"])[:, :s.lens[i]]


def _plain_causal(s, q, k, v, at):
    """Rows of one sequence, the last of its keys among them, into s.out and s.lse from row `at` on."""
    hkv, m, d = k.shape
    n, g = q.shape[1], q.shape[0] // hkv
    k, v = k.float().unsqueeze(1), v.float().unsqueeze(1)
    step = max(1, (1 << 29) // (q.shape[0] * m))  # rows at once: their scores fill 2 GB at most
    for a in range(0, n, step):
        b = min(n, a + step)
        last = m - n + b  # no row of these sees more
        x = torch.matmul(q[:, a:b].float().reshape(hkv, g, b - a, d), k[:, :, :last].transpose(2, 3)) * s.scale
        key = torch.arange(last, device=x.device)[None]
        x = x.masked_fill(key > torch.arange(m - n + a, last, device=x.device)[:, None], -math.inf)
        top = x.amax(dim=3, keepdim=True)
        p = torch.exp(x - top)
        total = p.sum(dim=3, keepdim=True)
        o = torch.matmul(p, v[:, :, :last]) / total
        s.out[:, at + a:at + b] = o.reshape(hkv * g, b - a, d).to(s.dt)
        s.lse[:, at + a:at + b] = (top + total.log()).reshape(hkv * g, b - a)


def _plain_padded(s):
    """All sequences at once, their keys and their new tokens padded to the longest."""
    c = s.case
    hq, hkv, d, n_seq, page = c["hq"], c["hkv"], c["d"], c["n_seq"], c["page"]
    most, g, dev = max(s.new), c["hq"] // c["hkv"], s.table.device
    lens, first = s.lens_dev.long(), s.cu[:-1].long()
    count = s.cu[1:].long() - first
    t = torch.arange(most, device=dev)
    rows = first[:, None] + torch.minimum(t[None], count[:, None] - 1)                   # [n_seq, most]
    q = s.q[:, rows].float().permute(1, 0, 2, 3).reshape(n_seq, hkv, g * most, d)
    k, v = (x[s.table.long()].float().transpose(1, 2).reshape(n_seq, hkv, -1, d) for x in (s.k_pages, s.v_pages))
    x = torch.matmul(q, k.transpose(2, 3)).view(n_seq, hkv, g, most, -1) * s.scale
    seen = (lens - count)[:, None] + torch.minimum(t[None], count[:, None] - 1)          # the row's own slot
    x = x.masked_fill((torch.arange(x.shape[-1], device=dev) > seen[:, :, None])[:, None, None], -math.inf)
    top = x.amax(dim=4, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(dim=4, keepdim=True)
    o = torch.matmul(p.view(n_seq, hkv, g * most, -1), v).view(n_seq, hq, most, d) / total.view(n_seq, hq, most, 1)
    l = (top + total.log()).view(n_seq, hq, most)
    s.out[:, rows.reshape(-1)] = o.transpose(0, 1).reshape(hq, n_seq * most, d).to(s.dt)
    s.lse[:, rows.reshape(-1)] = l.transpose(0, 1).reshape(hq, n_seq * most)


def _slots(s):
    """Sequence and slot of every new token."""
    first = s.cu[:-1].long()
    count = s.cu[1:].long() - first
    i = torch.arange(s.q.shape[1], device=s.cu.device)
    seq = torch.searchsorted(s.cu[1:].long(), i, right=True)
    return seq, s.lens_dev.long()[seq] - count[seq] + i - first[seq]


def _rotated(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), dim=-1).flatten(-2) if interleaved else torch.cat((a, b), dim=-1)
    return torch.cat((turned, y[..., rot:]), dim=-1).to(x.dtype)


def _plain_append(s):
    c = s.case
    seq, slot = _slots(s)
    angle = (slot if s.pos is None else s.pos).double()[:, None] * s.inv_freq.double()[None]
    cos, sin = angle.cos().float(), angle.sin().float()
    at = s.table[seq, slot // c["page"]].long()
    row = slot % c["page"]
    s.k_pages[at, :, row] = _rotated(s.k, cos, sin, c["interleaved"]).transpose(0, 1)
    s.v_pages[at, :, row] = s.v.transpose(0, 1)
    s.q_out.copy_(_rotated(s.q, cos, sin, c["interleaved"]))


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    starts = [sum(s.new[:i]) for i in range(len(s.new))]
    if case["op"] == "append":
        # complex numbers turned by exp(i angle), token by token of a sequence, written page by page
        half = case["rot"] // 2
        pairs = [(2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half) for i in range(half)]
        re, im = [p[0] for p in pairs], [p[1] for p in pairs]
        pages = {"k": s.k_pages.double(), "v": s.v_pages.double()}
        q_out = s.q.double().contiguous()
        for i, (a, n, m) in enumerate(zip(starts, s.new, s.lens)):
            slots = torch.arange(m - n, m, device=s.q.device)
            turn = slots.double() if s.pos is None else s.pos[a:a + n].double()
            unit = torch.polar(torch.ones((), dtype=torch.float64, device=s.q.device).expand(n, half),
                               torch.outer(turn, s.inv_freq.double()))

            def turned(x):
                y = x[:, a:a + n].double().clone()
                z = torch.complex(y[..., re], y[..., im]) * unit
                y[..., re], y[..., im] = z.real, z.imag
                return y

            q_out[:, a:a + n] = turned(s.q)
            where = (s.table[i].long()[slots // case["page"]], slots % case["page"])
            pages["k"][where[0], :, where[1]] = turned(s.k).transpose(0, 1)
            pages["v"][where[0], :, where[1]] = s.v[:, a:a + n].double().transpose(0, 1)
        return {"k_pages": pages["k"], "v_pages": pages["v"], "q": q_out}
    hq, group = case["hq"], case["hq"] // case["hkv"]
    out = torch.empty(s.out.shape, dtype=torch.float64, device=s.q.device)
    lse = torch.empty(s.lse.shape, dtype=torch.float64, device=s.q.device)
    for i, (a, n, m) in enumerate(zip(starts, s.new, s.lens)):
        if case["op"] == "prefill":
            k, v = s.k[:, a:a + n], s.v[:, a:a + n]
        else:
            slots = torch.arange(m, device=s.q.device)
            which, row = s.table[i].long()[slots // case["page"]], slots % case["page"]
            k, v = s.k_pages[which, :, row].transpose(0, 1), s.v_pages[which, :, row].transpose(0, 1)
        kd, vd = k.double(), v.double()
        rows = max(1, (1 << 27) // m)
        for h in range(hq):
            for b in range(0, n, rows):
                e = min(n, b + rows)
                w = (s.q[h, a + b:a + e].double() @ kd[h // group].T) * s.scale
                w = w + torch.triu(torch.full_like(w, -math.inf), diagonal=m - n + b + 1)
                l = torch.logsumexp(w, dim=1)
                lse[h, a + b:a + e] = l
                out[h, a + b:a + e] = torch.exp(w - l[:, None]) @ vd[h // group]
    return {"out": out, "lse": lse}
