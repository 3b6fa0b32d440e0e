"""A small decoder served with continuous batching: the attention operators and the expert-cached MoE layer together.

    python examples/serve_decoder.py [--layers 4] [--requests 12] [--new 24] [--w4]

Random weights, random prompts, greedy answers.  Every step is one packed batch: running requests bring one token each, prompts
come in chunks, requests that do not get pages wait, finished ones give theirs back.  Per step the page bookkeeping runs once
(``FtAttn.slots``); per layer: projection, ``FtAttn.qk_rope`` into the layer's cache, ``FtAttn.forward``, output projection, router
and ``FtMoe.layer`` over the host pool of experts.  The host only reads back the answers and who was admitted.

With ``--w4`` the projections and the output head have 4-bit weights with group scales (``FtDense.w4``), residual and norm between the blocks
are one call (``FtDense.add_norm``), and the answers come with their log probabilities and the entropy (``FtDense.logprobs``).
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_16157_b200 import attention as A      # noqa: E402
from paper_2608_16157_b200 import binding as B        # noqa: E402
from paper_2608_16157_b200 import dense as D          # noqa: E402
from paper_2608_16157_b200 import workload as W       # noqa: E402

EPS = 1e-6


def quantise(w, group=64):
    """4-bit codes, two in a byte, and group scales of a [k, n] matrix, as ``FtDense.w4_pack`` takes them ([n, k / 2], [n, k / group])."""
    g = w.float().t().contiguous().view(w.shape[1], -1, group)
    scales = (g.abs().amax(-1) / 7).clamp(min=1e-8).to(w.dtype)
    q = (g / scales.float()[..., None]).round().clamp(-8, 7).add(8).to(torch.uint8).reshape(w.shape[1], -1)
    return (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), scales


class Decoder:
    """Weights, expert pool, caches and handles of an L-layer decoder; :meth:`step` runs one packed batch."""

    def __init__(self, *, layers=2, shape=W.TINY, n_q_heads=4, n_kv_heads=2, head_dim=64, vocab=512, page_tokens=16, n_pages=64,
                 max_requests=8, max_tokens=128, max_pages=32, expert_slots=4, rope_base=1e6, seed=0, device="cuda:0", w4=False):
        self.L, self.shape, self.vocab, self.dev = layers, shape, vocab, torch.device(device)
        self.hq, self.hkv, self.d = n_q_heads, n_kv_heads, head_dim
        g = torch.Generator(device=self.dev)
        g.manual_seed(seed)
        rand = lambda *s, scale: (torch.randn(*s, generator=g, device=self.dev) * scale).bfloat16()
        hid, width = shape.d, (n_q_heads + 2 * n_kv_heads) * head_dim
        self.embed, self.head = rand(vocab, hid, scale=1.0), rand(hid, vocab, scale=hid ** -0.5)
        self.w_qkv = [rand(hid, width, scale=hid ** -0.5) for _ in range(layers)]
        self.w_o = [rand(n_q_heads * head_dim, hid, scale=(n_q_heads * head_dim) ** -0.5) for _ in range(layers)]
        self.w_q = [1 + rand(head_dim, scale=0.2) for _ in range(layers)]
        self.w_k = [1 + rand(head_dim, scale=0.2) for _ in range(layers)]
        self.router = [torch.randn(hid, shape.n_experts, generator=g, device=self.dev) * hid ** -0.5 for _ in range(layers)]
        # rotation table, queries, caches
        freq = rope_base ** (-torch.arange(0, head_dim, 2, device=self.dev, dtype=torch.float64) / head_dim)
        ang = torch.arange(max_pages * page_tokens, device=self.dev, dtype=torch.float64)[:, None] * freq
        self.cos_sin = torch.cat([ang.cos(), ang.sin()], 1).float()
        cfg = A.make_config(n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, page_tokens=page_tokens, n_pages=n_pages,
                            max_requests=max_requests, max_tokens=max_tokens, max_pages=max_pages)
        self.attn = A.FtAttn(cfg)
        self.cache = [torch.zeros(n_pages, 2, n_kv_heads, page_tokens, head_dim, dtype=torch.bfloat16, device=self.dev) for _ in range(layers)]
        # experts: all of them in pinned host memory, `expert_slots` a layer in HBM
        self.pool = B.HostPool(layers * shape.n_experts * shape.expert_bytes)
        W.fill_pool(self.pool.tensor, shape, layers, seed)
        self.moe = B.FtMoe(B.make_config(hidden=hid, inter=shape.inter, n_experts=shape.n_experts, top_k=shape.top_k, n_layers=layers,
                                         slots_per_layer=expert_slots, max_tokens=max_tokens, host_pool_ptr=self.pool.ptr.value,
                                         host_pool_bytes=self.pool.n_bytes, fill_mode=B.FT_FILL_SM))
        # page bookkeeping; counts alternate between two buffers
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=self.dev)
        self.table = i32(max_requests, max_pages)
        self.free_pages = torch.arange(n_pages, dtype=torch.int32, device=self.dev)
        self.n_free, self.n_free_next = torch.tensor([n_pages], dtype=torch.int32, device=self.dev), i32(1)
        self.ctx, self.ctx_next = i32(max_requests), i32(max_requests)
        self.q_start, self.admitted = i32(max_requests + 1), i32(max_requests)
        # with 4-bit weights: the handle, the matrices laid out once
        self.dense = None
        if w4:
            self.dense = D.FtDense(self.dev.index)
            pack = lambda w: self.dense.w4_pack(*quantise(w))
            self.w4_qkv, self.w4_o, self.w4_head = [pack(w) for w in self.w_qkv], [pack(w) for w in self.w_o], pack(self.head)
            self.answer_logprob = self.answer_entropy = None       # of the latest step's answers
        self.record = None          # a list: (layer, attention input, attention output) of every step go there

    def close(self):
        self.attn.destroy()
        self.moe.destroy()
        if self.dense is not None:
            self.dense.destroy()
        self.pool.free()

    @staticmethod
    def _norm(x):
        f = x.float()
        return (f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)).to(x.dtype)

    def step(self, new_len, tokens):
        """One packed batch: ``new_len`` of every request row (< 0: finished), ``tokens`` of all rows in order.  Returns
        (answer of every row's last token, admitted) on the host."""
        t, hq, hkv, d = len(tokens), self.hq, self.hkv, self.d
        new = torch.tensor(new_len, dtype=torch.int32, device=self.dev)
        position = torch.empty(t, dtype=torch.int32, device=self.dev)
        slot = torch.empty_like(position)
        self.attn.slots(new, self.ctx, self.table, self.free_pages, self.n_free, max(max(new_len), 0), q_start=self.q_start,
                        kv_len=self.ctx_next, n_free_out=self.n_free_next, admitted=self.admitted, position=position, slot=slot)
        self.ctx, self.ctx_next = self.ctx_next, self.ctx
        self.n_free, self.n_free_next = self.n_free_next, self.n_free
        if t == 0:
            return [0] * len(new_len), self.admitted.tolist()
        x = self.embed[torch.tensor(tokens, device=self.dev)]
        q_rot, out = (torch.empty(t, hq, d, dtype=torch.bfloat16, device=self.dev) for _ in range(2))
        y = torch.empty_like(x)
        if self.dense is not None:
            return self._step_w4(new_len, t, x, y, q_rot, out, position, slot)
        for layer in range(self.L):
            h = self._norm(x)
            qkv = h @ self.w_qkv[layer]
            self.attn.qk_rope(qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
                              qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)), q_rot, self.cache[layer], position, slot, self.cos_sin,
                              w_q=self.w_q[layer], w_k=self.w_k[layer], eps=EPS)
            self.attn.forward(q_rot, self.cache[layer], self.table, out)
            if self.record is not None:
                self.record.append((layer, h.clone(), out.clone()))
            x = x + out.flatten(1) @ self.w_o[layer]
            h = self._norm(x)
            self.moe.layer(layer, h.float() @ self.router[layer], h, y, t)
            x = x + y
        last = (self.q_start[1:len(new_len) + 1].long() - 1).clamp(min=0)
        answers = (self._norm(x[last]) @ self.head).float().argmax(-1)
        both = torch.stack([answers.to(torch.int32), self.admitted[:len(new_len)]]).tolist()     # one read back
        return both[0], both[1]


    def _step_w4(self, new_len, t, x, y, q_rot, out, position, slot):
        """The same with 4-bit weights: x is the residual stream, y the output of the block at hand."""
        n, hq, hkv, d, dense = len(new_len), self.hq, self.hkv, self.d, self.dense
        h = torch.empty_like(x)
        qkv = torch.empty(t, (hq + 2 * hkv) * d, dtype=x.dtype, device=self.dev)
        for layer in range(self.L):
            dense.add_norm(y if layer else None, x, x, h, eps=EPS)
            dense.w4(h, self.w4_qkv[layer], qkv)
            self.attn.qk_rope(qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
                              qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)), q_rot, self.cache[layer], position, slot, self.cos_sin,
                              w_q=self.w_q[layer], w_k=self.w_k[layer], eps=EPS)
            self.attn.forward(q_rot, self.cache[layer], self.table, out)
            if self.record is not None:
                self.record.append((layer, h.clone(), out.clone()))
            dense.w4(out.flatten(1), self.w4_o[layer], y)
            dense.add_norm(y, x, x, h, eps=EPS)
            self.moe.layer(layer, h.float() @ self.router[layer], h, y, t)
        dense.add_norm(y, x, None, h, eps=EPS)
        last = (self.q_start[1:n + 1].long() - 1).clamp(min=0)
        logits = torch.empty(n, self.vocab, device=self.dev)
        dense.w4(h[last], self.w4_head, logits)
        answers = torch.empty(n, 1, dtype=torch.int32, device=self.dev)
        self.answer_logprob, self.answer_entropy = torch.empty(n, 1, device=self.dev), torch.empty(n, device=self.dev)
        dense.logprobs(logits, entropy=self.answer_entropy, top_ids=answers, top_logprobs=self.answer_logprob)
        both = torch.stack([answers[:, 0], self.admitted[:n]]).tolist()
        return both[0], both[1]


def serve(dec, prompts, n_new, chunk=48, log=None):
    """Serves all prompts with the decoder's request rows; returns the answers of each.

    Pages go by the requests' age (their order): while one waits for pages, younger ones bring no tokens, and if it cannot go on
    although it is alone, the youngest gives its pages back and starts again later.  So the oldest always gets on, and all end."""
    cfg = dec.attn.cfg
    if n_new < 1 or not all(prompts):
        raise ValueError("a request needs a prompt and at least one answer")
    if any(-(-(len(p) + n_new - 1) // cfg.page_tokens) > min(cfg.n_pages, cfg.max_pages) for p in prompts):
        raise ValueError("a request does not fit the page pool or its row of the block table")
    waiting, answers = list(range(len(prompts))), [[] for _ in prompts]
    run = [None] * cfg.max_requests          # [request, tokens given so far]; "done": pages go back in the next step
    blocked = None                           # the oldest request that got no pages in the last step
    while waiting or any(r is not None for r in run):
        for i, r in enumerate(run):
            if r is None and waiting:
                run[i] = [waiting.pop(0), 0]
        active = sorted((r[0], i) for i, r in enumerate(run) if r is not None and r != "done")
        take, text, left = [0] * len(run), [[]] * len(run), cfg.max_tokens
        for request, i in active:
            if blocked is not None and request > blocked:
                break
            rest = (list(prompts[request]) + answers[request])[run[i][1]:]
            take[i] = min(len(rest), chunk, left)
            text[i] = rest[:take[i]]
            left -= take[i]
        new_len = [-1 if r == "done" else n for r, n in zip(run, take)]
        got, admitted = dec.step(new_len, sum(text, []))
        waits = [request for request, i in active if take[i] and not admitted[i]]
        if log:
            log(f"step: {sum(n > 0 for n in take)} requests, {sum(take)} tokens, {run.count('done')} finished, {len(waits)} wait for pages")
        run = [None if r == "done" else r for r in run]
        for request, i in active:
            if take[i] and admitted[i]:
                run[i][1] += take[i]
                if run[i][1] == len(prompts[request]) + len(answers[request]):
                    answers[request].append(got[i])
                    if len(answers[request]) == n_new:
                        run[i] = "done"
        blocked = min(waits, default=None)
        if waits and sum(n > 0 for n in take) == 1:
            last, i = max((request, i) for request, i in active if request == blocked or run[i][1])
            if last == blocked:
                raise RuntimeError("pages are missing from the pool")
            waiting.insert(0, last)
            answers[last] = []
            run[i] = "done"
    return answers


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--new", type=int, default=24)
    ap.add_argument("--w4", action="store_true", help="4-bit projections and output head")
    args = ap.parse_args()
    rng = np.random.default_rng(0)
    dec = Decoder(layers=args.layers, n_pages=40, w4=args.w4)
    prompts = [rng.integers(0, dec.vocab, int(rng.integers(1, 150))).tolist() for _ in range(args.requests)]
    answers = serve(dec, prompts, args.new, log=print)
    for p, a in zip(prompts[:4], answers):
        print(f"prompt of {len(p)} tokens -> {a}")
    assert dec.attn.sync_status() == 0 and dec.moe.sync_status() == 0
    assert int(dec.n_free) == 40              # every page came back
    if dec.dense is not None:
        print("dense kernels:", dec.dense.launch_count(), " status:", dec.dense.sync_status())
    print("attention-side kernels:", dec.attn.launch_count(), " MoE kernels:", dec.moe.launch_count())
    dec.close()


if __name__ == "__main__":
    main()
