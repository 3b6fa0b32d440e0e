"""Plain 64-bit forms of the attention-side operators on the CPU, and the error bounds their tests use."""
from __future__ import annotations

import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
# relative error of one rounding to nearest: 2^-8 for an 8-bit significand, 2^-11 for an 11-bit one
UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def ceil_div(a, b):
    return -(-a // b)


def slots(new_len, ctx_len, table, free, n_free, page, rows):
    """Sequential definition of a step's bookkeeping.  Returns a dict of numpy arrays."""
    table, free = table.copy(), free.copy()
    top = n_free
    for r, n in enumerate(new_len):
        if n < 0:
            for b in range(ceil_div(ctx_len[r], page)):
                free[top] = table[r, b]
                top += 1
    q_start, kv, adm = [0], [], []
    pos, slot = np.full(rows, -1, np.int32), np.full(rows, -1, np.int32)
    wanted = 0
    for r, n in enumerate(new_len):
        n_tok = max(n, 0)
        q_start.append(q_start[-1] + n_tok)
        if n < 0:
            kv.append(0)
            adm.append(0)
            continue
        held = ceil_div(ctx_len[r], page)
        need = ceil_div(ctx_len[r] + n, page) - held
        wanted += need
        if need > 0 and wanted > n_free + sum(ceil_div(c, page) for c, m in zip(ctx_len, new_len) if m < 0):
            kv.append(ctx_len[r])
            adm.append(0)
            continue
        for b in range(need):
            top -= 1
            table[r, held + b] = free[top]
        for i in range(n):
            p = ctx_len[r] + i
            pos[q_start[r] + i] = p
            slot[q_start[r] + i] = table[r, p // page] * page + p % page
        kv.append(ctx_len[r] + n)
        adm.append(1)
    i32 = lambda x: np.asarray(x, np.int32)
    return dict(table=table, free=free, n_free=i32([top]), q_start=i32(q_start), kv_len=i32(kv), admitted=i32(adm), position=pos, slot=slot)


def norm_rope(x, w, cos_sin, position, eps, interleaved):
    """x [T, H, D] -> float64 result and the magnitudes (|a| + |b| of each rotated pair) that scale its float error."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    y, mag = x.clone(), x.abs()
    if cos_sin is not None:
        half = cos_sin.shape[1] // 2
        cs = cos_sin.double()[position.long().clamp(min=0)]
        cos, sin = cs[:, None, :half], cs[:, None, half:]
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
        mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


def attention(q, cache, table, q_start, kv_len, page, window, scale):
    """float64 (out, lse, sum of weights times |v|, sum of |v|) of every packed row; rows that see nothing: 0, -inf."""
    t, hq, d = q.shape
    hkv = cache.shape[2]
    out = torch.zeros(t, hq, d, dtype=torch.float64)
    lse = torch.full((t, hq), -float("inf"), dtype=torch.float64)
    wabs, vabs = torch.zeros_like(out), torch.zeros_like(out)
    for r in range(len(kv_len)):
        n, l = int(q_start[r + 1] - q_start[r]), int(kv_len[r])
        for i in range(n):
            p = l - n + i
            lo = max(0, p - window + 1) if window else 0
            if p < 0:
                continue
            j = torch.arange(lo, p + 1)
            pages = table[r].long()[j // page]
            k = cache[pages, 0, :, j % page].double().permute(1, 2, 0)           # [hkv, d, keys]
            v = cache[pages, 1, :, j % page].double().permute(1, 0, 2)
            row = int(q_start[r]) + i
            s = (q[row].double().view(hkv, hq // hkv, d) @ k) * scale
            w = torch.softmax(s, -1)
            out[row] = (w @ v).reshape(hq, d)
            wabs[row] = (w @ v.abs()).reshape(hq, d)
            vabs[row] = v.abs().sum(1)[:, None].expand(hkv, hq // hkv, d).reshape(hq, d)
            lse[row] = torch.logsumexp(s, -1).reshape(hq)
    return out, lse, wabs, vabs


def attention_bound(dtype, ref, wabs, vabs, score_max):
    """Largest error of an output element: one rounding of the result, one rounding of every softmax weight to the
    operand type of the second product (its sum is kept unrounded), weights below the smallest number of the type
    (2^-25 of the largest, fp16 only), and 2^-16 of the weights for float scores (D terms of relative error 2^-24 in a
    score of magnitude score_max), exponentials and sums."""
    u = UNIT[dtype]
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0
    return u * ref.abs() + u * (1 + u) * wabs + tiny * vabs + 2.0 ** -16 * (1.0 + score_max) * wabs + 1e-30
