"""Plain 64-bit forms of the operators of ``dense`` and the error bounds their tests use."""
from __future__ import annotations

import torch

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# half a step of the type, relative; below fp16's normal numbers half a step is 2^-25
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25, torch.float32: 1e-38}


def rounding(ref, dtype):
    return UNIT[dtype] * ref.abs() + TINY[dtype]


def add_norm(y, res, gate, w_post, w_pre, *, post, w_offset, eps, res_scale, y_scale):
    """float64 (r', h) and bounds of their float errors: every elementwise step is off by 2^-24, a mean of d <= 16384 squares by at most
    (16 + 10) * 2^-24 (16 in a thread, then a tree), its root by half of that plus 2^-22: below 2^-19 in all."""
    f = 2.0 ** -19
    u = mag = None
    if y is not None:
        u = y.double()
        if post:
            u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps)
            if w_post is not None:
                u = u * (w_offset + w_post.double())
        if gate is not None:
            u = u * gate.double()
        u = y_scale * u
    r = torch.zeros_like(u) if res is None else res_scale * res.double()
    mag = r.abs() + (0 if u is None else u.abs())
    r = r if u is None else r + u
    e_r = f * mag
    inv = 1 / torch.sqrt((r * r).mean(-1, keepdim=True) + eps)
    w = torch.ones(r.shape[-1], dtype=torch.float64, device=r.device) if w_pre is None else w_offset + w_pre.double()
    h = r * inv * w
    e_h = e_r * inv * w.abs() + h.abs() * (e_r.pow(2).mean(-1, keepdim=True).sqrt() * inv + f)
    return r, h, e_r, e_h


def w4_weights(codes, scales, zeros):
    """float64 [n, k]."""
    n, groups = scales.shape
    q = torch.stack([codes & 15, codes >> 4], -1).reshape(n, groups, -1).double()
    z = 8.0 if zeros is None else zeros.double()[..., None]
    return ((q - z) * scales.double()[..., None]).reshape(n, -1)


def w4(x, w, bias, out_dtype):
    """float64 result and a bound of its error before the result is rounded.  Up to 16 tokens, and for float results: products are exact; a group's
    sum goes through at most 8 tensor-core instructions of 16 products, each off by 2^-22 of the magnitudes (aligned and cut), and is added in
    float: at most k / 32 groups, 16 warps and 8 blocks.  More tokens with 16-bit results: every weight is rounded once to the type (half a step,
    2^-25 below fp16's normal numbers), and the tensor core adds k / 16 times, each off by 2^-22 at most."""
    ref = x.double() @ w.t()
    mag = x.double().abs() @ w.abs().t()
    if bias is not None:
        ref, mag = ref + bias.double(), mag + bias.double().abs()
    err = (2.0 ** -19 + (x.shape[1] / 32 + 24) * 2.0 ** -24) * mag
    if x.shape[0] > 16 and out_dtype is not torch.float32:
        err = (UNIT[x.dtype] + x.shape[1] / 16 * 2.0 ** -22) * mag + TINY[x.dtype] * x.double().abs().sum(-1, keepdim=True)
    return ref, err


def logprobs(logits, scale, k):
    """float64 (log probabilities of all, entropy, ids, bound of a log probability's float error, bound of the entropy's).  Rows without a
    distribution: NaN; rows of nothing: -infinity, 0, -1.  Errors: an exponent (x - m) c is off by 2^-22 of itself, an exponential by 2^-22, a sum
    by its longest chain (the pieces of one of 512 threads and 30 joins)."""
    x = logits.double() * scale
    t, v = x.shape
    bad = torch.isnan(x).any(-1) | (x == float("inf")).any(-1)
    none = (x == -float("inf")).all(-1) & ~bad
    safe = torch.where((bad | none)[:, None], 0.0, x)
    logp = torch.log_softmax(safe, -1)
    p = logp.exp()
    dist = torch.where(torch.isinf(safe), 0.0, safe.amax(-1, keepdim=True) - safe)     # distance from the largest
    ent = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    mean = (p * dist).sum(-1, keepdim=True)
    chain = (v / 512 + 64) * 2.0 ** -24
    e_logp = 2.0 ** -21 * (1 + dist + mean) + chain * (1 + mean)
    e_ent = (2.0 ** -20 * (1 + mean) + 2 * chain * (1 + mean))[:, 0] + 2.0 ** -21 * (p * dist * dist).sum(-1)
    logp = torch.where(none[:, None], -float("inf"), logp)
    logp = torch.where(bad[:, None], float("nan"), logp)
    ent = torch.where(bad, float("nan"), torch.where(none, 0.0, ent))
    key = torch.where(torch.isnan(logits), -float("inf"), logits.double())
    order = torch.sort(key, dim=-1, descending=True, stable=True)
    ids = order.indices[:, :k]
    ids = torch.where(order.values[:, :k] == -float("inf"), -1, ids)
    ids = torch.where(bad[:, None], -1, ids)
    if ids.shape[1] < k:
        ids = torch.nn.functional.pad(ids, (0, k - ids.shape[1]), value=-1)
    return logp, ent, ids, e_logp, e_ent
