"""The serving example end to end: chunked prompts, single tokens, requests that wait for pages and pages that come back, all
operators in their places, against attention computed without pages."""
import numpy as np
import pytest
import torch

from examples import serve_decoder as S
from tests import attn_reference as R

pytestmark = pytest.mark.gpu


def test_served_batches_equal_attention_without_pages():
    rng = np.random.default_rng(3)
    dec = S.Decoder(layers=2, n_pages=10, max_requests=4, max_tokens=64, max_pages=8, seed=3)
    prompts = [rng.integers(0, dec.vocab, n).tolist() for n in (70, 1, 33, 50, 17, 40)]
    # every step's inputs and outputs of the attention, and which rows belong to which request's positions
    log = []
    inner = dec.step

    def step(new_len, tokens):
        dec.record = []
        got = inner(new_len, tokens)
        q_start = np.concatenate([[0], np.cumsum(np.maximum(new_len, 0))])
        log.append((list(new_len), q_start, list(got[1]), [(l, h.cpu(), o.cpu()) for l, h, o in dec.record]))
        return got

    dec.step = step
    answers = S.serve(dec, prompts, n_new=6, chunk=24)
    assert all(len(a) == 6 for a in answers)
    assert dec.attn.sync_status() == 0 and dec.moe.sync_status() == 0
    assert int(dec.n_free) == 10 and sorted(dec.free_pages.tolist()) == list(range(10))
    assert any(n > 0 and not a for new, _, adm, _ in log for n, a in zip(new, adm)), "the case has to make a request wait"
    hq, hkv, d = dec.hq, dec.hkv, dec.d
    table = dec.cos_sin.cpu()
    for layer in range(dec.L):
        w = dec.w_qkv[layer].cpu().double()
        past = [None] * 4                       # per request row: keys and values so far
        err2 = ref2 = 0.0
        for new, q_start, adm, rec in log:
            for r, n in enumerate(new):
                if n < 0:
                    past[r] = None
                if n <= 0 or not adm[r]:
                    continue
                _, h, out = rec[layer]
                rows = slice(int(q_start[r]), int(q_start[r + 1]))
                qkv = (h[rows].double() @ w).bfloat16()      # (the projection's own rounding)
                start = 0 if past[r] is None else past[r][0].shape[0]
                pos = torch.arange(start, start + n)
                q, k, v = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)), qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
                q = R.norm_rope(q, dec.w_q[layer].cpu(), table, pos, S.EPS, False)[0].bfloat16().double()
                k = R.norm_rope(k, dec.w_k[layer].cpu(), table, pos, S.EPS, False)[0].bfloat16().double()
                past[r] = (k, v.double()) if past[r] is None else (torch.cat([past[r][0], k]), torch.cat([past[r][1], v.double()]))
                kk, vv = (z.repeat_interleave(hq // hkv, 1) for z in past[r])
                s = torch.einsum("thd,jhd->htj", q, kk) * d ** -0.5
                s = s.masked_fill(torch.arange(kk.shape[0])[None, :] > pos[:, None], -float("inf"))
                want = torch.einsum("htj,jhd->thd", torch.softmax(s, -1), vv)
                err2 += float((out[rows].double() - want).pow(2).sum())
                ref2 += float(want.pow(2).sum())
        # roundings of the result (2^-9 on average) and of the weights, and single-ulp flips of q, k, v: below 1e-2
        assert (err2 / ref2) ** 0.5 <= 1e-2
    dec.close()
