"""What a decoder's step has besides its attention and its experts, as measured workloads.

Three operators, each with its plain form in elementary torch operations:

``norm``   a block's output joins the residual stream: norm after the block, gate, residual scale, norm before the next block
``w4``     products with 4-bit weights and group scales: projections and output head, from single tokens to prompt chunks
``logp``   log probabilities of given tokens, entropy and the most likely alternatives from the logits

A case is a dict of plain values; all data come from the seed of :func:`prepare`.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a small decode batch between two blocks: the call is all latency
        dict(name="norm_decode_8", op="norm", dtype="bf16", res="bf16", tokens=8, d=2048, post=False, gate="none", pad=0),
        # a prompt chunk of a decoder with norms on both sides of its blocks, gated per element, float residual stream, odd width
        dict(name="norm_sandwich_1021", op="norm", dtype="fp16", res="fp32", tokens=1021, d=1537, post=True, gate="element", pad=7),
        # a whole prefill step; the block's output is scaled per channel
        dict(name="norm_prefill_16384", op="norm", dtype="bf16", res="bf16", tokens=16384, d=2048, post=True, gate="channel", pad=0),

        # q/k/v projection of one token: latency
        dict(name="w4_qkv_1", op="w4", dtype="bf16", out="same", tokens=1, k=2048, n=5120, group=128, zeros=False, bias=True),
        # output projection of a decode batch, small groups, zero points
        dict(name="w4_out_8", op="w4", dtype="fp16", out="same", tokens=8, k=4096, n=2048, group=32, zeros=True, bias=False),
        # output head of a few requests, float logits: the weights stream from HBM
        dict(name="w4_head_5", op="w4", dtype="bf16", out="fp32", tokens=5, k=2048, n=150001, group=64, zeros=False, bias=False),
        # a full decode batch through a wide projection
        dict(name="w4_batch_64", op="w4", dtype="bf16", out="same", tokens=64, k=7168, n=7168, group=128, zeros=False, bias=False),
        # a prompt chunk through the same projection: bound by the products
        dict(name="w4_chunk_4096", op="w4", dtype="bf16", out="same", tokens=4096, k=7168, n=7168, group=128, zeros=True, bias=False),

        # one user's next token, float logits, an odd vocabulary
        dict(name="logp_one", op="logp", dtype="fp32", tokens=1, vocab=50001, given=1, top=20, masked=0.0, pad=0),
        # a decode batch; half of the vocabulary masked out by a grammar
        dict(name="logp_decode_8", op="logp", dtype="bf16", tokens=8, vocab=150000, given=1, top=5, masked=0.5, pad=0),
        # scoring of several labels at every position of a text, padded rows
        dict(name="logp_labels_515", op="logp", dtype="fp16", tokens=515, vocab=32003, given=7, top=20, masked=0.0, pad=29),
        # log probabilities of a whole prompt chunk
        dict(name="logp_prompt_2048", op="logp", dtype="bf16", tokens=2048, vocab=150000, given=1, top=8, masked=0.0, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    cap = {}
    for c in listed():
        w = work(c)
        b, f = cap.get(c["op"], (0, 0))
        cap[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    op = rng.choice(["norm", "norm", "w4", "w4", "w4", "w4", "logp", "logp"])
    few = rng.random() < 0.6
    while True:
        dtype = rng.choice(["bf16", "fp16"])
        if op == "norm":
            c = dict(op="norm", dtype=dtype, res=rng.choice([dtype, "fp32"]), tokens=_log(rng, 1, 16384),
                     d=rng.choice([_log(rng, 64, 8192), 8 * _log(rng, 8, 1024), 1024, 2048, 4096, 7168]), post=rng.random() < 0.5,
                     gate=rng.choice(["none", "element", "channel", "token"]), pad=rng.choice([0, 0, 0, 8, 5]))
        elif op == "w4":
            group = rng.choice([32, 64, 128, 128])
            c = dict(op="w4", dtype=dtype, out=rng.choice(["same", "same", "fp32"]), tokens=_log(rng, 1, 64) if few else _log(rng, 1, 4096),
                     k=rng.choice([group * _log(rng, max(1, 256 // group), 8192 // group), 2048, 4096, 7168]),
                     n=rng.choice([_log(rng, 100, 150001), 16 * _log(rng, 16, 1024), 5120, 2048, 7168]), group=group, zeros=rng.random() < 0.4,
                     bias=rng.random() < 0.3)
        else:
            c = dict(op="logp", dtype=rng.choice(["bf16", "fp16", "fp32"]), tokens=_log(rng, 1, 64) if few else _log(rng, 1, 2048),
                     vocab=rng.choice([_log(rng, 1000, 150000), 8 * _log(rng, 125, 18750)]), given=rng.choice([1, 1, rng.randint(2, 16)]),
                     top=rng.choice([1, rng.randint(2, 32)]), masked=rng.choice([0.0, 0.0, rng.uniform(0.1, 0.9)]), pad=rng.choice([0, 0, rng.randint(1, 64)]))
        w = work(c)
        b, f = cap[op]
        if w["bytes"] <= b and w["flops"] <= f:
            return c


def _size(dtype):
    return 4 if dtype == "fp32" else 2


def work(case):
    if case["op"] == "norm":
        t, d, e, r = case["tokens"], case["d"], _size(case["dtype"]), _size(case["res"])
        gate = {"none": 0, "element": t * d, "channel": d, "token": t}[case["gate"]]
        return {"bytes": t * d * (2 * e + 2 * r) + e * (gate + d + (d if case["post"] else 0)), "flops": t * d * (6 + (3 if case["post"] else 0))}
    if case["op"] == "w4":
        t, n, k = case["tokens"], case["n"], case["k"]
        groups = n * (k // case["group"])
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": n * k // 2 + groups * 2 + (groups // 2 if case["zeros"] else 0) + 2 * t * k + out * t * n + (2 * n if case["bias"] else 0),
                "flops": 2 * t * n * k}
    t, v = case["tokens"], case["vocab"]
    return {"bytes": t * v * _size(case["dtype"]) + t * (8 * case["given"] + 4 + 8 * case["top"]), "flops": 6 * t * v}


# ------------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _handle():
    from paper_2608_16157_b200 import dense
    return dense.FtDense()


def _prepare_norm(case, seed):
    g, dt, rt = _gen(seed), DTYPES[case["dtype"]], DTYPES[case["res"]]
    t, d, pad = case["tokens"], case["d"], case["pad"]
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    # the stream has grown over the layers before and holds a few channels of large magnitude
    big = 1.0 + 20.0 * (torch.rand(d, generator=g, device="cuda") < 0.004)
    gate = {"none": None, "element": lambda: rand(t, d), "channel": lambda: 1 + 0.3 * rand(1, d), "token": lambda: rand(t, 1)}[case["gate"]]
    st = dict(case=case, op="norm", y=rand(t, d + pad).to(dt)[:, :d], res=(3.0 * big * rand(t, d)).to(rt),
              gate=None if gate is None else gate().to(dt), w_pre=(0.3 * rand(d)).to(dt), w_post=(0.3 * rand(d)).to(dt) if case["post"] else None,
              res_scale=0.9, y_scale=0.7, res_out=torch.empty(t, d, dtype=rt, device="cuda"), out=torch.empty(t, d, dtype=dt, device="cuda"))
    if own:
        st["dense"] = _handle()
    return st


def _prepare_w4(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    t, n, k, group = (case[i] for i in ("tokens", "n", "k", "group"))
    # codes of normally distributed weights, two in a byte, the even index in the low half
    codes = torch.empty(n, k // 2, dtype=torch.uint8, device="cuda")
    for i in range(0, n, 16384):
        m = min(16384, n - i)
        half = lambda: torch.randn(m, k // 2, generator=g, device="cuda").mul_(2.6).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
        codes[i:i + m] = half() | (half() << 4)
    scales = ((0.5 + torch.rand(n, k // group, generator=g, device="cuda")) * (0.4 * k ** -0.5)).to(dt)
    zeros = torch.randint(6, 11, (n, k // group), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    bias = torch.randn(n, generator=g, device="cuda").to(dt) if case["bias"] else None
    big = 1.0 + 10.0 * (torch.rand(k, generator=g, device="cuda") < 0.01)
    st = dict(case=case, op="w4", x=(big * torch.randn(t, k, generator=g, device="cuda")).to(dt), bias=bias,
              y=torch.empty(t, n, dtype=dt if case["out"] == "same" else torch.float32, device="cuda"))
    if own:
        # the weights are laid out once, when a program loads them
        st["dense"] = _handle()
        st["w"] = st["dense"].w4_pack(codes, scales, zeros)
    else:
        st.update(codes=codes, scales=scales, zeros=zeros)
    return st


def _prepare_logp(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    t, v = case["tokens"], case["vocab"]
    # a frequency of every word and a context's own preferences; some rows are nearly certain
    prior = -0.8 * torch.log1p(torch.randperm(v, generator=g, device="cuda").float())
    sharp = 1.0 + 3.0 * torch.rand(t, 1, generator=g, device="cuda")
    logits = torch.empty(t, v + case["pad"], dtype=dt, device="cuda")
    tokens = torch.empty(t, case["given"], dtype=torch.int32, device="cuda")
    for i in range(0, t, 256):
        m = min(256, t - i)
        x = (torch.randn(m, v, generator=g, device="cuda") + 0.4 * prior) * sharp[i:i + m]
        if case["masked"]:
            x.masked_fill_(torch.rand(m, v, generator=g, device="cuda") < case["masked"], float("-inf"))
        logits[i:i + m, :v] = x.to(dt)
        logits[i:i + m, v:] = float("nan")
        # given tokens: likely ones, as those of a text or of an answer
        tokens[i:i + m] = torch.multinomial(torch.softmax(x / sharp[i:i + m], -1), case["given"], generator=g).to(torch.int32)
    f32 = lambda *s: torch.empty(*s, dtype=torch.float32, device="cuda")
    st = dict(case=case, op="logp", logits=logits[:, :v], tokens=tokens, scale=0.8, logprob=f32(t, case["given"]), entropy=f32(t),
              top_ids=torch.empty(t, case["top"], dtype=torch.int32, device="cuda"), top_logprobs=f32(t, case["top"]))
    if own:
        st["dense"] = _handle()
    return st


def prepare(case, seed):
    return {"norm": _prepare_norm, "w4": _prepare_w4, "logp": _prepare_logp}[case["op"]](case, seed)


# -------------------------------------------------------------------------------------------------------- plain forms
def _rms(x):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _plain_norm(s):
    u = s["y"].float()
    if s["w_post"] is not None:
        u = _rms(u) * (1.0 + s["w_post"].float())
    if s["gate"] is not None:
        u = u * s["gate"].float()
    r = s["res_scale"] * s["res"].float() + s["y_scale"] * u
    s["out"].copy_(_rms(r) * (1.0 + s["w_pre"].float()))
    s["res_out"].copy_(r)
    return dict(res=s["res_out"], out=s["out"])


def _plain_w4(s):
    k, group = s["case"]["k"], s["case"]["group"]
    x = s["x"].float()
    step = max(1, (1 << 28) // k)
    for i in range(0, s["codes"].shape[0], step):
        c = s["codes"][i:i + step]
        q = torch.stack([c & 15, c >> 4], -1).view(c.shape[0], k // group, group).float()
        z = 8.0 if s["zeros"] is None else s["zeros"][i:i + step].float()[..., None]
        w = ((q - z) * s["scales"][i:i + step].float()[..., None]).view(c.shape[0], k)
        y = torch.matmul(x, w.t())
        if s["bias"] is not None:
            y = y + s["bias"][i:i + step].float()
        s["y"][:, i:i + step] = y
    return s["y"]


def _plain_logp(s):
    n = s["top_ids"].shape[1]
    rows = max(1, (1 << 27) // s["logits"].shape[1])
    for i in range(0, s["logits"].shape[0], rows):
        raw = s["logits"][i:i + rows].float()
        x = raw * s["scale"]
        x = x - x.amax(-1, keepdim=True)
        e = torch.exp(x)
        total = e.sum(-1, keepdim=True)
        lse = torch.log(total)
        s["logprob"][i:i + rows] = torch.gather(x, 1, s["tokens"][i:i + rows].long()) - lse
        s["entropy"][i:i + rows] = (lse - (e * x.clamp(min=-1e30)).sum(-1, keepdim=True) / total)[:, 0]
        order = torch.sort(raw, dim=-1, descending=True, stable=True).indices[:, :n]      # (equal ones: the lowest index first)
        s["top_ids"][i:i + rows] = order.to(torch.int32)
        s["top_logprobs"][i:i + rows] = torch.gather(x, 1, order) - lse
    return dict(logprob=s["logprob"], entropy=s["entropy"], top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])


# ---------------------------------------------------------------------------------------------------------------- run
def run(s):
    if not own:
        return {"norm": _plain_norm, "w4": _plain_w4, "logp": _plain_logp}[s["op"]](s)
    a = s["dense"]
    if s["op"] == "norm":
        a.add_norm(s["y"], s["res"], s["res_out"], s["out"], post=s["w_post"] is not None, w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"],
                   w_offset=1.0, eps=EPS, res_scale=s["res_scale"], y_scale=s["y_scale"])
        return dict(res=s["res_out"], out=s["out"])
    if s["op"] == "w4":
        a.w4(s["x"], s["w"], s["y"], bias=s["bias"])
        return s["y"]
    a.logprobs(s["logits"], tokens=s["tokens"], logprob=s["logprob"], entropy=s["entropy"], top_ids=s["top_ids"], top_logprobs=s["top_logprobs"],
               scale=s["scale"])
    return dict(logprob=s["logprob"], entropy=s["entropy"], top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])


# -------------------------------------------------------------------------------------------------------------- exact
def _exact_norm(s):
    def norm(x, w):
        return x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS) * (w.double() + 1)

    u = s["y"].double()
    if s["case"]["post"]:
        u = norm(u, s["w_post"])
    if s["gate"] is not None:
        u = s["gate"].double() * u
    r = torch.add(u * s["y_scale"], s["res"].double(), alpha=s["res_scale"])
    return dict(res=r, out=norm(r, s["w_pre"]))


def _exact_w4(s):
    n, k, group = (s["case"][i] for i in ("n", "k", "group"))
    x = s["x"].double()
    out = torch.empty(x.shape[0], n, dtype=torch.float64, device="cuda")
    # codes and zero points apart: the sum over codes, minus zero point times the group's sum of x
    even, odd = x[:, 0::2], x[:, 1::2]
    sums = x.view(x.shape[0], k // group, group).sum(-1)
    step = max(1, (1 << 26) // k)
    for i in range(0, n, step):
        c, sc = s["codes"][i:i + step], s["scales"][i:i + step].double()
        per = sc.repeat_interleave(group // 2, 1)
        y = even @ (torch.remainder(c, 16).double() * per).t() + odd @ (torch.div(c, 16, rounding_mode="floor").double() * per).t()
        z = torch.full_like(sc, 8.0) if s["zeros"] is None else s["zeros"][i:i + step].double()
        y -= sums @ (sc * z).t()
        out[:, i:i + step] = y if s["bias"] is None else y + s["bias"][i:i + step].double()
    return out


def _exact_logp(s):
    t, v = s["logits"].shape
    lp, ent, ids, top = [], [], [], []
    k = s["case"]["top"]
    rows = max(1, (1 << 26) // v)
    for i in range(0, t, rows):
        raw = s["logits"][i:i + rows].double()
        logp = torch.log_softmax(raw * s["scale"], -1)
        lp.append(logp.gather(1, s["tokens"][i:i + rows].long()))
        ent.append(-torch.where(torch.isinf(logp), 0.0, logp.exp() * logp).sum(-1))
        left, got = raw.clone(), []
        for _ in range(k):             # the largest left, the first of equals
            best = left.amax(-1, keepdim=True)
            at = torch.where(left == best, torch.arange(v, device="cuda"), v).amin(-1, keepdim=True)
            got.append(at)
            left.scatter_(1, at, -math.inf)
        at = torch.cat(got, 1)
        ids.append(at.to(torch.int32))
        top.append(logp.gather(1, at))
    return dict(logprob=torch.cat(lp), entropy=torch.cat(ent), top_ids=torch.cat(ids), top_logprobs=torch.cat(top))


def exact(case, seed):
    global own
    was, own = own, False          # the inputs as they are, not laid out
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "w4": _exact_w4, "logp": _exact_logp}[case["op"]](s)
