"""The operators around the expert-cached MoE layer in a serving step, as measured workloads.

Three operators of the attention side of a decoder layer, each with its plain form in elementary torch operations:

``slots``  block tables and slot maps of a step from the request lengths (page allocation and release, positions, slots)
``rope``   RMS norm of every query and key head, position rotation, write of keys and values into the paged cache
``attn``   causal attention of the step's new tokens over the paged cache (single tokens, chunks, whole prompts)

A case is a dict of plain values.  The lengths of a case's requests follow from its ``lengths`` number alone, so the work
of a case is known without its data; all values come from the seed of :func:`prepare`.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a small decode batch: the call is all latency
        dict(name="slots_decode_8", op="slots", requests=8, ctx=2000, chunks=0, chunk=0, finished=0, page=16, spare=64, lengths=11),
        # continuous batching: mostly single tokens, some prompts in chunks, some requests just finished, pages run out
        dict(name="slots_mixed_250", op="slots", requests=250, ctx=4000, chunks=9, chunk=509, finished=12, page=16, spare=-100, lengths=12),
        # a prefill step: 63 prompts of which each brings a chunk
        dict(name="slots_prefill_63", op="slots", requests=63, ctx=3000, chunks=63, chunk=260, finished=0, page=64, spare=400, lengths=13),

        # decode batch of the 30B-A3B-shaped decoder (32 query and 4 key/value heads of 128)
        dict(name="rope_decode_8", op="rope", dtype="bf16", hq=32, hkv=4, d=128, rot=128, interleaved=False, tokens=8, page=16, qkv_pad=0, norm=True),
        # an odd chunk with small heads, half of each rotated, interleaved pairs, a fused projection with padded rows
        dict(name="rope_chunk_1021", op="rope", dtype="fp16", hq=64, hkv=8, d=64, rot=32, interleaved=True, tokens=1021, page=32, qkv_pad=64, norm=True),
        # a whole prefill step
        dict(name="rope_prefill_16384", op="rope", dtype="bf16", hq=32, hkv=4, d=128, rot=128, interleaved=False, tokens=16384, page=64, qkv_pad=0, norm=True),

        # one user, short context: latency
        dict(name="attn_decode_1", op="attn", dtype="bf16", hq=32, hkv=4, d=128, page=16, window=0, requests=1, ctx=1000, ragged=0.0, new=1, chunks=0, chunk=0, lengths=21),
        # the decode batch of the framework's benchmark, ragged contexts
        dict(name="attn_decode_8", op="attn", dtype="bf16", hq=32, hkv=4, d=128, page=16, window=0, requests=8, ctx=6000, ragged=0.6, new=1, chunks=0, chunk=0, lengths=22),
        # a full decode batch over long contexts: the cache streams from HBM
        dict(name="attn_decode_128", op="attn", dtype="bf16", hq=32, hkv=4, d=128, page=64, window=0, requests=128, ctx=12000, ragged=0.7, new=1, chunks=0, chunk=0, lengths=23),
        # verification of drafted tokens: a few tokens per request, sliding window, small heads
        dict(name="attn_draft_33", op="attn", dtype="fp16", hq=64, hkv=8, d=64, page=32, window=2048, requests=33, ctx=6000, ragged=0.9, new=5, chunks=0, chunk=0, lengths=24),
        # chunked prefill beside running decodes
        dict(name="attn_mixed_32", op="attn", dtype="bf16", hq=32, hkv=4, d=128, page=16, window=0, requests=32, ctx=7000, ragged=0.8, new=1, chunks=1, chunk=515, lengths=25),
        # a long prompt from an empty cache
        dict(name="attn_prefill_16384", op="attn", dtype="bf16", hq=32, hkv=4, d=128, page=64, window=0, requests=1, ctx=0, ragged=0.0, new=1, chunks=1, chunk=16384, lengths=26),
    ]


HEADS = [(32, 4, 128), (64, 8, 64), (16, 16, 128), (28, 4, 128), (40, 8, 128), (24, 8, 64), (64, 4, 128), (10, 10, 64)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    cap = {}
    for c in listed():
        w = work(c)
        b, f = cap.get(c["op"], (0, 0))
        cap[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    kind = rng.choice(["slots", "rope", "rope", "attn_decode", "attn_decode", "attn_draft", "attn_mixed", "attn_prefill"])
    while True:
        hq, hkv, d = rng.choice(HEADS)
        page = rng.choice([16, 32, 64, 128])
        heads = dict(dtype=rng.choice(["bf16", "fp16"]), hq=hq, hkv=hkv, d=d, page=page)
        seed = rng.randrange(1 << 30)
        window = rng.choice([0, 0, 0, _log(rng, 100, 8000)])
        if kind == "slots":
            r = _log(rng, 1, 256)
            c = dict(op="slots", requests=r, ctx=_log(rng, 1, 16000), chunks=rng.randint(0, r), chunk=_log(rng, 2, max(2, 16384 // r)),
                     finished=rng.randint(0, r // 4), page=page, spare=rng.choice([_log(rng, 1, 2000), -_log(rng, 1, 200)]), lengths=seed)
        elif kind == "rope":
            rot = rng.choice([d, d, d // 2])
            c = dict(op="rope", rot=rot, interleaved=rng.random() < 0.5, tokens=_log(rng, 1, 16384), qkv_pad=rng.choice([0, 0, 64]),
                     norm=rng.random() < 0.8, **heads)
        elif kind == "attn_decode":
            c = dict(op="attn", window=window, requests=_log(rng, 1, 256), ctx=_log(rng, 1, 100000), ragged=rng.uniform(0.0, 1.0), new=1,
                     chunks=0, chunk=0, lengths=seed, **heads)
        elif kind == "attn_draft":
            c = dict(op="attn", window=window, requests=_log(rng, 1, 128), ctx=_log(rng, 10, 50000), ragged=rng.uniform(0.0, 1.0),
                     new=rng.randint(2, 12), chunks=0, chunk=0, lengths=seed, **heads)
        elif kind == "attn_mixed":
            r = _log(rng, 2, 128)
            c = dict(op="attn", window=window, requests=r, ctx=_log(rng, 50, 30000), ragged=rng.uniform(0.0, 1.0), new=1,
                     chunks=rng.randint(1, min(r, 4)), chunk=_log(rng, 16, 2048), lengths=seed, **heads)
        else:
            c = dict(op="attn", window=window, requests=rng.randint(1, 4), ctx=0, ragged=0.0, new=1, chunks=4, chunk=_log(rng, 16, 16384),
                     lengths=seed, **heads)
            c["chunks"] = c["requests"]
        w = work(c)
        b, f = cap[c["op"]]
        if w["bytes"] <= b and w["flops"] <= f and w["flops"] + w["bytes"] > 0:
            return c


# ------------------------------------------------------------------------------------------------- lengths of a case
def _slot_lengths(case):
    """(new_len, ctx_len) of every request; -1 marks a finished request."""
    rng = random.Random(case["lengths"])
    n_req, kinds = case["requests"], []
    kinds += ["finished"] * case["finished"]
    kinds += ["chunk"] * min(case["chunks"], n_req - len(kinds))
    kinds += ["single"] * (n_req - len(kinds))
    rng.shuffle(kinds)
    new, ctx = [], []
    for k in kinds:
        c = rng.randint(0, case["ctx"])
        if k == "finished":
            new.append(-1)
        elif k == "chunk":
            new.append(rng.randint(max(1, case["chunk"] // 2), case["chunk"]))
            c = c // 2
        else:
            new.append(1)
        ctx.append(c)
    return new, ctx


def _attn_lengths(case):
    """(new_len, kv_len) of every request; kv_len counts the new tokens."""
    rng = random.Random(case["lengths"])
    new, kv = [], []
    for r in range(case["requests"]):
        c = int(round(case["ctx"] * (1.0 - case["ragged"] * rng.random())))
        n = case["new"]
        if r < case["chunks"]:
            n = case["chunk"] if r == 0 else rng.randint(max(1, case["chunk"] // 2), case["chunk"])
        new.append(n)
        kv.append(c + n)
    order = list(range(case["requests"]))
    rng.shuffle(order)
    return [new[i] for i in order], [kv[i] for i in order]


def _ceil(a, b):
    return -(-a // b)


def work(case):
    if case["op"] == "slots":
        new, ctx = _slot_lengths(case)
        p = case["page"]
        tokens = sum(max(n, 0) for n in new)
        need = sum(max(0, _ceil(c + n, p) - _ceil(c, p)) for n, c in zip(new, ctx) if n >= 0)
        freed = sum(_ceil(c, p) for n, c in zip(new, ctx) if n < 0)
        first = sum(1 for n, c in zip(new, ctx) if n > 0 and c % p)
        return {"bytes": 8 * len(new) + 8 + 12 * len(new) + 8 * tokens + 8 * need + 8 * freed + 4 * first, "flops": 4 * tokens}
    if case["op"] == "rope":
        t, d = case["tokens"], case["d"]
        heads = case["hq"] + 2 * case["hkv"]
        return {"bytes": 2 * (2 * t * heads * d) + 8 * t + 4 * t * case["rot"] + (4 * d if case["norm"] else 0),
                "flops": t * (case["hq"] + case["hkv"]) * (3 * case["rot"] + (4 * d if case["norm"] else 0))}
    new, kv = _attn_lengths(case)
    w = case["window"] or (1 << 40)
    pairs = keys = 0
    for n, l in zip(new, kv):
        lo = l - n                                   # positions lo .. l-1 attend min(position + 1, w) keys each
        full = max(0, min(l, w) - lo)                # rows that see every key before them
        pairs += full * lo + full * (full + 1) // 2 + (n - full) * min(w, l)
        keys += l - max(0, lo + 1 - w)
    d = case["d"]
    return {"bytes": 2 * 2 * sum(new) * case["hq"] * d + 2 * 2 * keys * case["hkv"] * d + 4 * _ceil(keys, case["page"]),
            "flops": 4 * d * case["hq"] * pairs}


# ------------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _handle(case, **kw):
    from paper_2608_16157_b200 import attention
    return attention.FtAttn(attention.make_config(page_tokens=case["page"], **kw))


def _prepare_slots(case, seed):
    g = _gen(seed)
    new, ctx = _slot_lengths(case)
    p, n_req = case["page"], len(new)
    tokens = sum(max(n, 0) for n in new)
    held = [_ceil(c, p) for c in ctx]
    need = [max(0, _ceil(c + n, p) - h) if n >= 0 else 0 for n, c, h in zip(new, ctx, held)]
    # free pages before the step: enough for all (spare > 0) or short by some (spare < 0)
    n_free = max(0, sum(need) - sum(h for n, h in zip(new, held) if n < 0) + case["spare"])
    n_pages = sum(held) + n_free + 8
    max_pages = max(max(h + e for h, e in zip(held, need)), 1)
    order = torch.randperm(n_pages, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    first = np.concatenate([[0], np.cumsum(held)])
    idx = np.full((n_req, max_pages), -1, dtype=np.int64)
    for r in range(n_req):
        idx[r, :held[r]] = np.arange(first[r], first[r + 1])
    idx = torch.from_numpy(idx).cuda()
    table = torch.where(idx >= 0, order[idx.clamp(min=0)], torch.full_like(idx, -1, dtype=torch.int32))
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_free] = order[int(first[-1]):int(first[-1]) + n_free]
    z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    st = dict(case=case, op="slots", new_len=_i32(new), ctx_len=_i32(ctx), table=table, free_pages=free, n_free=_i32([n_free]), tokens=tokens,
              max_new=max(max(new), 0), n_pages=n_pages, q_start=z(n_req + 1), kv_len=z(n_req), n_free_out=z(1), admitted=z(n_req),
              position=z(tokens), slot=z(tokens))
    if own:
        st["attn"] = _handle(case, n_q_heads=32, n_kv_heads=4, head_dim=128, n_pages=n_pages, max_requests=n_req, max_tokens=max(tokens, 1),
                             max_pages=max_pages)
    return st


def _prepare_rope(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    t, hq, hkv, d, p, rot = (case[k] for k in ("tokens", "hq", "hkv", "d", "page", "rot"))
    width = (hq + 2 * hkv) * d + case["qkv_pad"]
    # one fused projection of the step's tokens; q, k and v are views of its rows
    qkv = (torch.randn(t, width, generator=g, device="cuda") * 1.5).to(dt)
    n_pages = _ceil(t, p) + 3
    pages = torch.randperm(n_pages, generator=g, device="cuda")[:_ceil(t, p)]
    off = torch.arange(t, device="cuda")
    slot = (pages[off // p] * p + off % p).to(torch.int32)
    max_pos = 32768
    base = int(torch.randint(0, max_pos - t, (1,), generator=g, device="cuda"))
    freq = 1e6 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    ang = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * freq
    weight = lambda: (1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt) if case["norm"] else None
    st = dict(case=case, op="rope", q=qkv[:, :hq * d].unflatten(1, (hq, d)), k=qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
              v=qkv[:, (hq + hkv) * d:(hq + 2 * hkv) * d].unflatten(1, (hkv, d)), position=(off + base).to(torch.int32), slot=slot,
              w_q=weight(), w_k=weight(), cos_sin=torch.cat([ang.cos(), ang.sin()], 1).float(),
              q_out=torch.empty(t, hq, d, dtype=dt, device="cuda"),
              kv_cache=torch.randn(n_pages, 2, hkv, p, d, generator=g, device="cuda").to(dt))
    if own:
        st["attn"] = _handle(case, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_pages=n_pages, max_requests=1, max_tokens=t, max_pages=n_pages,
                             dtype=case["dtype"])
    return st


def _prepare_attn(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    hq, hkv, d, p = (case[k] for k in ("hq", "hkv", "d", "page"))
    new, kv = _attn_lengths(case)
    n_req, t = len(new), sum(new)
    held = [_ceil(l, p) for l in kv]
    n_pages, max_pages = sum(held) + 4, max(held)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    first = np.concatenate([[0], np.cumsum(held)])
    idx = np.full((n_req, max_pages), -1, dtype=np.int64)
    for r in range(n_req):
        idx[r, :held[r]] = np.arange(first[r], first[r + 1])
    idx = torch.from_numpy(idx).cuda()
    table = torch.where(idx >= 0, order[idx.clamp(min=0)], torch.full_like(idx, -1, dtype=torch.int32))
    # heads as they come out of the norm: unit mean square times a learned weight; some keys draw much attention
    cache = torch.empty(n_pages, 2, hkv, p, d, dtype=dt, device="cuda")
    for i in range(0, n_pages, 4096):
        n = min(4096, n_pages - i)
        kk = torch.randn(n, hkv, p, d, generator=g, device="cuda")
        kk *= 1.0 + (torch.rand(n, hkv, p, 1, generator=g, device="cuda") < 0.01) * 1.0
        cache[i:i + n, 0] = kk.to(dt)
        cache[i:i + n, 1] = (0.7 * torch.randn(n, hkv, p, d, generator=g, device="cuda")).to(dt)
    st = dict(case=case, op="attn", q=(1.2 * torch.randn(t, hq, d, generator=g, device="cuda")).to(dt), kv_cache=cache, table=table, new=new, kv=kv,
              q_start=_i32([0] + list(np.cumsum(new))), kv_len=_i32(kv), out=torch.empty(t, hq, d, dtype=dt, device="cuda"))
    if own:
        st["attn"] = _handle(case, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_pages=n_pages, max_requests=n_req, max_tokens=t,
                             max_pages=max_pages, dtype=case["dtype"], window=case["window"])
    return st


def prepare(case, seed):
    return {"slots": _prepare_slots, "rope": _prepare_rope, "attn": _prepare_attn}[case["op"]](case, seed)


# -------------------------------------------------------------------------------------------------------- plain forms
def _plain_slots(s):
    p, tok = s["case"]["page"], s["tokens"]
    new, ctx, table, free, n_pages = s["new_len"], s["ctx_len"], s["table"], s["free_pages"], s["n_pages"]
    col = torch.arange(table.shape[1], device="cuda")
    finished = new < 0
    n = new.clamp(min=0)
    held = (ctx + p - 1) // p
    n_freed = torch.where(finished, held, 0)
    ends = torch.cumsum(n_freed, 0)
    # finished requests push their pages; what must not be written goes to a place past the end
    stack = torch.cat([free, free.new_full((1,), -1)])
    dst = (s["n_free"] + ends - n_freed)[:, None] + col
    dst = torch.where(finished[:, None] & (col < held[:, None]), dst, n_pages).clamp(max=n_pages)
    stack[dst] = table
    avail = s["n_free"] + ends[-1]
    need = torch.where(finished, 0, (ctx + n + p - 1) // p - held)
    incl = torch.cumsum(need, 0)
    admitted = ~finished & ((need == 0) | (incl <= avail))
    k = col - held[:, None]
    fresh = admitted[:, None] & (k >= 0) & (k < need[:, None])
    src = (avail - 1 - (incl - need))[:, None] - k
    table.copy_(torch.where(fresh, stack[src.clamp(0, n_pages)], table))
    free.copy_(stack[:n_pages])
    q_start = torch.cat([n.new_zeros(1), torch.cumsum(n, 0)]).to(torch.int32)
    t = torch.arange(tok, device="cuda")
    r = (torch.searchsorted(q_start, t, right=True) - 1).clamp(0, n.numel() - 1)
    pos = ctx[r] + (t - q_start[r])
    ok = admitted[r]
    slot = table[r, (pos // p).clamp(max=table.shape[1] - 1)] * p + pos % p
    return dict(table=table, free_pages=free, n_free=(avail - torch.where(admitted, need, 0).sum()).to(torch.int32), q_start=q_start,
                kv_len=torch.where(finished, 0, torch.where(admitted, ctx + n, ctx)).to(torch.int32), admitted=admitted.to(torch.int32),
                position=torch.where(ok, pos, -1).to(torch.int32), slot=torch.where(ok, slot, -1).to(torch.int32))


def _plain_heads(x, w, cos, sin, interleaved):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    half = cos.shape[-1]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2] = a * cos - b * sin
        y[..., 1:2 * half:2] = b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half] = a * cos - b * sin
        y[..., half:2 * half] = b * cos + a * sin
    return y


def _plain_rope(s):
    c = s["case"]
    p, half = c["page"], c["rot"] // 2
    cs = s["cos_sin"][s["position"].long()]
    cos, sin = cs[:, None, :half], cs[:, None, half:]
    slot = s["slot"].long()
    s["q_out"].copy_(_plain_heads(s["q"], s["w_q"], cos, sin, c["interleaved"]))
    s["kv_cache"][slot // p, 0, :, slot % p] = _plain_heads(s["k"], s["w_k"], cos, sin, c["interleaved"]).to(s["kv_cache"].dtype)
    s["kv_cache"][slot // p, 1, :, slot % p] = s["v"]
    return dict(q=s["q_out"], kv_cache=s["kv_cache"])


def _plain_attn(s):
    c = s["case"]
    hq, hkv, d, p, window = c["hq"], c["hkv"], c["d"], c["page"], c["window"]
    group, scale, t0 = hq // hkv, c["d"] ** -0.5, 0
    for r, (n, l) in enumerate(zip(s["new"], s["kv"])):
        start = l - n
        lo_page = max(0, start + 1 - window) // p if window else 0
        pages = s["table"][r, lo_page:_ceil(l, p)].long()
        kv = s["kv_cache"][pages]                                                        # [pages, 2, hkv, p, d]
        kv = kv.permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :l - lo_page * p].float()
        key = torch.arange(lo_page * p, l, device="cuda")
        step = max(1, min(n, (1 << 28) // max(1, hq * key.numel())))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = s["q"][t0 + i:t0 + i + m].float().view(m, hkv, group, d).permute(1, 2, 0, 3).reshape(hkv, group * m, d)
            x = torch.matmul(q, kv[0].transpose(1, 2)) * scale
            pos = start + i + torch.arange(m, device="cuda")
            hide = key[None, :] > pos[:, None]
            if window:
                hide = hide | (key[None, :] <= pos[:, None] - window)
            x = x.view(hkv, group, m, -1).masked_fill_(hide, float("-inf"))
            x = torch.exp(x - x.amax(-1, keepdim=True))
            x = x / x.sum(-1, keepdim=True)
            o = torch.matmul(x.view(hkv, group * m, -1), kv[1])
            s["out"][t0 + i:t0 + i + m] = o.view(hkv, group, m, d).permute(2, 0, 1, 3).reshape(m, hq, d).to(s["out"].dtype)
        t0 += n
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------- run
def run(s):
    if not own:
        return {"slots": _plain_slots, "rope": _plain_rope, "attn": _plain_attn}[s["op"]](s)
    a = s["attn"]
    if s["op"] == "slots":
        a.slots(s["new_len"], s["ctx_len"], s["table"], s["free_pages"], s["n_free"], s["max_new"], q_start=s["q_start"], kv_len=s["kv_len"],
                n_free_out=s["n_free_out"], admitted=s["admitted"], position=s["position"], slot=s["slot"])
        return dict(table=s["table"], free_pages=s["free_pages"], n_free=s["n_free_out"], q_start=s["q_start"], kv_len=s["kv_len"],
                    admitted=s["admitted"], position=s["position"], slot=s["slot"])
    if s["op"] == "rope":
        a.qk_rope(s["q"], s["k"], s["v"], s["q_out"], s["kv_cache"], s["position"], s["slot"], s["cos_sin"], w_q=s["w_q"], w_k=s["w_k"], eps=EPS,
                  interleaved=s["case"]["interleaved"])
        return dict(q=s["q_out"], kv_cache=s["kv_cache"])
    # the work partition of these lengths is made in the call, as for the first layer of a step
    a.plan(s["q_start"], s["kv_len"], s["q"].shape[0], max(s["new"]))
    a.forward(s["q"], s["kv_cache"], s["table"], s["out"])
    return s["out"]


# -------------------------------------------------------------------------------------------------------------- exact
def _exact_slots(s):
    p = s["case"]["page"]
    new, ctx = s["new_len"].tolist(), s["ctx_len"].tolist()
    table, stack = s["table"].cpu().numpy().copy(), s["free_pages"].cpu().numpy().copy()
    top = int(s["n_free"][0])
    for r, n in enumerate(new):
        if n < 0:
            for b in range(_ceil(ctx[r], p)):
                stack[top] = table[r, b]
                top += 1
    q_start, kv_len, admitted, position, slot, wanted, taken = [0], [], [], [], [], 0, 0
    for r, n in enumerate(new):
        q_start.append(q_start[-1] + max(n, 0))
        if n < 0:
            kv_len.append(0)
            admitted.append(0)
            continue
        held = _ceil(ctx[r], p)
        need = _ceil(ctx[r] + n, p) - held
        wanted += need
        ok = need == 0 or wanted <= top
        admitted.append(int(ok))
        if ok:
            for b in range(need):
                table[r, held + b] = stack[top - 1 - taken]
                taken += 1
        kv_len.append(ctx[r] + n if ok else ctx[r])
        for i in range(ctx[r], ctx[r] + n):
            position.append(i if ok else -1)
            slot.append(int(table[r, i // p]) * p + i % p if ok else -1)
    return dict(table=torch.from_numpy(table).cuda(), free_pages=torch.from_numpy(stack).cuda(), n_free=_i32([top - taken]), q_start=_i32(q_start),
                kv_len=_i32(kv_len), admitted=_i32(admitted), position=_i32(position), slot=_i32(slot))


def _exact_rope(s):
    c = s["case"]
    half, d = c["rot"] // 2, c["d"]
    table = s["cos_sin"].double()[s["position"].long()]
    # the rotation as a complex product
    phase = torch.complex(table[:, :half], table[:, half:])[:, None]
    first = torch.arange(half, device="cuda") * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else half)

    def head(x, w):
        x = x.double()
        if w is not None:
            x = w.double() * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + EPS)
        z = torch.complex(x[..., first], x[..., second]) * phase
        x = x.clone()
        x[..., first], x[..., second] = z.real, z.imag
        return x

    cache = s["kv_cache"].double()
    k, v = head(s["k"], s["w_k"]), s["v"].double()
    page, row = s["slot"].long() // c["page"], s["slot"].long() % c["page"]
    cache[page, 0, :, row], cache[page, 1, :, row] = k, v
    return dict(q=head(s["q"], s["w_q"]), kv_cache=cache)


def _exact_attn(s):
    c = s["case"]
    hq, hkv, d, p = c["hq"], c["hkv"], c["d"], c["page"]
    out, t0 = [], 0
    for r, (n, l) in enumerate(zip(s["new"], s["kv"])):
        j = torch.arange(l, device="cuda")
        rows = s["table"][r].long()[j // p]
        keys = s["kv_cache"][rows, 0, :, j % p].double()                                 # [l, hkv, d]
        vals = s["kv_cache"][rows, 1, :, j % p].double()
        step = max(1, (1 << 27) // (hq * l))
        for i in range(0, n, step):
            q = s["q"][t0 + i:t0 + min(n, i + step)].double()
            m = q.shape[0]
            x = torch.einsum("mhgd,lhd->hgml", q.view(m, hkv, hq // hkv, d), keys) / math.sqrt(d)
            dist = (l - n + i + torch.arange(m, device="cuda"))[:, None] - j
            seen = dist >= 0
            if c["window"]:
                seen &= dist < c["window"]
            x = torch.where(seen, x, -math.inf)
            w = torch.softmax(x, -1)
            out.append(torch.einsum("hgml,lhd->mhgd", w, vals).reshape(m, hq, d))
        t0 += n
    return torch.cat(out)


def exact(case, seed):
    global own
    was, own = own, False          # inputs only: no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"slots": _exact_slots, "rope": _exact_rope, "attn": _exact_attn}[case["op"]](s)
