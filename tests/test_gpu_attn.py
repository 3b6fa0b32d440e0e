"""GPU parity of the attention operators against their 64-bit definitions, and their refusals."""
import numpy as np
import pytest
import torch

from paper_2608_16157_b200 import attention as A
from paper_2608_16157_b200 import binding as B
from tests import attn_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device=DEV)


# ------------------------------------------------------------------------------------------------------------- slots
def run_slots(new, ctx, page, n_free, extra_pages=5, pad_rows=0, pad_cols=3, stride_pad=0, seed=0, max_new=None):
    rng = np.random.default_rng(seed)
    held = [R.ceil_div(c, page) for c in ctx]
    cols = max([R.ceil_div(c + max(n, 0), page) for c, n in zip(ctx, new)] + [1]) + pad_cols
    n_pages = sum(held) + n_free + extra_pages
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(new), cols), -7, np.int32)
    at = 0
    for r, h in enumerate(held):
        table[r, :h] = order[at:at + h]
        at += h
    free = np.full(n_pages, -9, np.int32)
    free[:n_free] = order[at:at + n_free]
    rows = sum(max(n, 0) for n in new) + pad_rows
    ref = R.slots(new, ctx, table, free, n_free, page, rows)
    h = A.FtAttn(A.make_config(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=page, n_pages=n_pages, max_requests=len(new),
                               max_tokens=max(rows, 1), max_pages=cols))
    wide = torch.full((len(new), cols + stride_pad), -7, dtype=torch.int32, device=DEV)
    wide[:, :cols] = torch.from_numpy(table)
    tab, fr = wide[:, :cols], i32(free)
    o = {n: torch.full((k,), -5, dtype=torch.int32, device=DEV) for n, k in
         (("q_start", len(new) + 1), ("kv_len", len(new)), ("n_free_out", 1), ("admitted", len(new)), ("position", rows), ("slot", rows))}
    for _ in range(2):          # the counts are not updated in place: a repeated call gives the same step
        h.slots(i32(new), i32(ctx), tab, fr, i32([n_free]), max(max(new), 0) if max_new is None else max_new, **o)
    assert h.sync_status() == 0
    got = dict(table=tab, free=fr, n_free=o.pop("n_free_out"), **o)
    for n, g in got.items():
        assert np.array_equal(g.cpu().numpy(), ref[n]), n
    if stride_pad:
        assert (wide[:, cols:] == -7).all()
    h.destroy()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_slots_mixed(page):
    run_slots([1, 7, 0, 130, 1, -1, 33, -1, 16, 1], [15, 0, 31, 64, 128, 200, 1, 0, 16, 1000], page, 40, pad_rows=3, stride_pad=5)


@pytest.mark.parametrize("n_free", [0, 1, 2, 5, 9, 30])
def test_slots_out_of_pages(n_free):
    """Requests that need nothing are admitted behind one that does not fit; released pages are handed out again."""
    run_slots([20, 1, 50, -1, 1, 0, 3, 1], [16, 5, 30, 40, 32, 7, 16, 31], 16, n_free)


def test_slots_single_and_all_finished():
    run_slots([1], [0], 16, 1)
    run_slots([1], [16], 16, 0)
    run_slots([-1, -1, -1], [100, 0, 17], 16, 4)
    run_slots([0], [0], 16, 0)


@pytest.mark.parametrize("n_req", [255, 256, 257, 1000, 1024])
def test_slots_many_requests(n_req):
    rng = np.random.default_rng(n_req)
    new = [int(x) for x in rng.choice([1, 1, 1, 0, -1, 17, 90], n_req)]
    ctx = [int(x) for x in rng.integers(0, 400, n_req)]
    run_slots(new, ctx, 16, int(rng.integers(100, 3000)), pad_rows=int(rng.integers(0, 50)))


def test_slots_bad_lengths_are_latched_and_skipped():
    h = A.FtAttn(A.make_config(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=32, max_requests=4, max_tokens=64, max_pages=4))
    tab, fr = i32(np.arange(16).reshape(4, 4)), i32(np.arange(32))
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    for new, ctx, nf in (([1, 9, 1, 1], [0, 0, 0, 0], 20), ([1, 1, 1, 1], [0, -3, 0, 0], 20), ([1, 1, 1, 1], [0, 64, 0, 0], 20),
                         ([5, 5, 5, 5], [0, 0, 0, 0], 20), ([1, 1, 1, 1], [0, 0, 0, 0], 33), ([-1, 1, 1, 1], [40, 0, 0, 0], 31)):
        o = dict(q_start=z(5), kv_len=z(4), n_free_out=z(1), admitted=z(4), position=z(8), slot=z(8))
        h.slots(i32(new), i32(ctx), tab, fr, i32([nf]), 5, **o)
        assert h.sync_status() == B.FT_ERR_INVALID_ARG and h.sync_status() == 0
        assert int(o["admitted"].sum()) < 4
    h.destroy()


# -------------------------------------------------------------------------------------------------------------- rope
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d,rot,inter,norm", [
    (32, 4, 128, 128, False, True), (8, 8, 128, 64, False, True), (7, 1, 64, 64, True, True), (6, 2, 64, 32, True, True),
    (5, 5, 128, 8, False, True), (4, 2, 64, 24, False, False), (9, 3, 128, 0, False, True), (2, 1, 64, 40, True, False)])
def test_qk_rope(dtype, hq, hkv, d, rot, inter, norm):
    dt = R.DT[dtype]
    g = torch.Generator().manual_seed(hq * 1000 + d + rot)
    page, n_pages = 16, 9
    for t, pad in ((1, 0), (37, 12)):
        width = (hq + 2 * hkv) * d + pad
        qkv = (torch.randn(t, width, generator=g) * torch.exp(torch.randn(t, 1, generator=g) * 3)).to(dt)
        if t > 4:
            qkv[3] = 0                                              # a row of zeros: eps alone in the norm
        cs = torch.randn(50, rot, generator=g) if rot else None      # any table: the operator does not assume cos^2 + sin^2 = 1
        pos = torch.randint(0, 50, (t,), generator=g, dtype=torch.int32)
        slot = torch.randperm(n_pages * page, generator=g)[:t].to(torch.int32)
        if t > 8:
            pos[5], slot[5] = -1, -1                                 # not admitted
            slot[7] = -1                                             # not cached
        w_q = (1 + 0.5 * torch.randn(d, generator=g)).to(dt) if norm else None
        w_k = (1 + 0.5 * torch.randn(d, generator=g)).to(dt) if norm else None
        cut = lambda x: (x[:, :hq * d].unflatten(1, (hq, d)), x[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
                         x[:, (hq + hkv) * d:(hq + 2 * hkv) * d].unflatten(1, (hkv, d)))
        h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=n_pages, max_requests=1, max_tokens=64,
                                   max_pages=4, dtype=dtype))
        old = torch.randn(n_pages, 2, hkv, page, d, generator=g).to(dt)
        q, k, v = cut(qkv)
        yq, mq = R.norm_rope(q, w_q, cs, pos, 1e-5, inter)
        yk, mk = R.norm_rope(k, w_k, cs, pos, 1e-5, inter)
        dev = lambda x: None if x is None else x.to(DEV)
        for in_place in (False, True):
            qd, kd, vd = cut(qkv.to(DEV))
            out = qd if in_place else torch.full((t, hq, d), 7.0, dtype=dt, device=DEV)
            cache = old.to(DEV)
            h.qk_rope(qd, kd, vd, out, cache, dev(pos), dev(slot), dev(cs), w_q=dev(w_q), w_k=dev(w_k), eps=1e-5, interleaved=inter)
            assert h.sync_status() == 0
            u = R.UNIT[dtype]
            # one rounding to the type (fp16: never finer than half its smallest number), float arithmetic on |a| + |b|
            bound = lambda y, m: u * y.abs() + 2.0 ** -20 * m + (2.0 ** -25 if dtype == "fp16" else 1e-38)
            got = out.double().cpu()
            want = yq * (pos >= 0)[:, None, None]
            fits = want.abs() < 60000 if dtype == "fp16" else torch.ones_like(want, dtype=torch.bool)
            assert ((got - want).abs() <= bound(yq, mq))[fits].all()
            gc = cache.cpu()
            touched = torch.zeros(n_pages, page, dtype=torch.bool)
            for i in range(t):
                if slot[i] < 0:
                    continue
                p, o = int(slot[i]) // page, int(slot[i]) % page
                touched[p, o] = True
                kk = gc[p, 0, :, o].double()
                ok = yk[i].abs() < 60000 if dtype == "fp16" else torch.ones_like(kk, dtype=torch.bool)
                assert ((kk - yk[i]).abs() <= bound(yk[i], mk[i]))[ok].all()
                assert torch.equal(gc[p, 1, :, o], v[i])
            keep = ~touched[:, None, None, :, None].expand_as(gc)
            assert torch.equal(gc[keep], old[keep])                  # nothing else in the cache changes
        h.destroy()


@pytest.mark.parametrize("dtype,hq,hkv,d,rot,inter,norm,t", [
    ("bf16", 32, 4, 128, 128, False, True, 1003), ("fp16", 64, 8, 64, 32, True, True, 1500), ("bf16", 3, 1, 64, 64, False, False, 15200),
    ("fp16", 96, 8, 128, 48, False, True, 700), ("bf16", 8, 8, 128, 0, False, True, 1700)])
def test_qk_rope_many_tokens(dtype, hq, hkv, d, rot, inter, norm, t):
    """Enough tokens for the kernel that brings whole tokens to shared memory; rows with padding between them."""
    dt, page = R.DT[dtype], 64
    g = torch.Generator().manual_seed(t)
    n_pages = R.ceil_div(t, page) + 2
    qkv = torch.randn(t, (hq + 2 * hkv) * d + 16, generator=g).to(dt)
    cs = torch.randn(300, rot, generator=g) if rot else None
    pos = torch.randint(0, 300, (t,), generator=g, dtype=torch.int32)
    slot = torch.randperm(n_pages * page, generator=g)[:t].to(torch.int32)
    pos[::7], slot[::7], slot[3::11] = -1, -1, -1
    w_q = (1 + 0.5 * torch.randn(d, generator=g)).to(dt) if norm else None
    w_k = (1 + 0.5 * torch.randn(d, generator=g)).to(dt) if norm else None
    cut = lambda x: (x[:, :hq * d].unflatten(1, (hq, d)), x[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
                     x[:, (hq + hkv) * d:(hq + 2 * hkv) * d].unflatten(1, (hkv, d)))
    dev = lambda x: None if x is None else x.to(DEV)
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=n_pages, max_requests=1, max_tokens=t,
                               max_pages=4, dtype=dtype))
    qd, kd, vd = cut(dev(qkv))
    out, cache = torch.full((t, hq, d), 7.0, dtype=dt, device=DEV), torch.full((n_pages, 2, hkv, page, d), 3.0, dtype=dt, device=DEV)
    h.qk_rope(qd, kd, vd, out, cache, dev(pos), dev(slot), dev(cs), w_q=dev(w_q), w_k=dev(w_k), eps=1e-5, interleaved=inter)
    assert h.sync_status() == 0
    q, k, v = cut(qkv)
    yq, mq = R.norm_rope(q, w_q, cs, pos, 1e-5, inter)
    yk, mk = R.norm_rope(k, w_k, cs, pos, 1e-5, inter)
    bound = lambda y, m: R.UNIT[dtype] * y.abs() + 2.0 ** -20 * m + (2.0 ** -25 if dtype == "fp16" else 1e-38)
    want = yq * (pos >= 0)[:, None, None]
    assert ((out.double().cpu() - want).abs() <= bound(yq, mq)).all()
    gc = cache.cpu().permute(0, 3, 1, 2, 4).reshape(n_pages * page, 2, hkv, d)
    kept = slot >= 0
    rows = gc[slot[kept].long()]
    assert ((rows[:, 0].double() - yk[kept]).abs() <= bound(yk[kept], mk[kept])).all()
    assert torch.equal(rows[:, 1], v[kept])
    other = torch.ones(n_pages * page, dtype=torch.bool)
    other[slot[kept].long()] = False
    assert (gc[other] == 3.0).all()
    h.destroy()


def test_qk_rope_bad_indices_are_latched_and_skipped():
    hq, hkv, d, page, n_pages = 4, 2, 64, 16, 3
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=n_pages, max_requests=1, max_tokens=8, max_pages=4))
    x = torch.randn(2, hq + 2 * hkv, d, device=DEV).bfloat16()
    cs = torch.randn(10, d, device=DEV)
    for pos, slot in (([0, 10], [0, 1]), ([0, 1], [0, 48])):
        cache = torch.zeros(n_pages, 2, hkv, page, d, device=DEV).bfloat16()
        h.qk_rope(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], torch.empty(2, hq, d, device=DEV).bfloat16(), cache, i32(pos), i32(slot), cs)
        assert h.sync_status() == B.FT_ERR_INVALID_ARG and h.sync_status() == 0
        assert cache[0, :, :, 0].abs().sum() > 0 and cache[0, :, :, 1:].abs().sum() == 0 and cache[1:].abs().sum() == 0
    h.destroy()


# --------------------------------------------------------------------------------------------------------- attention
def make_attn(dtype, hq, hkv, d, page, window, lens, seed=0, garbage=True, cols_pad=2, stride_pad=0, q_pad=0, amp=1.0):
    """Cache, table and queries on the CPU; what holds no token is NaN (or infinite)."""
    g = torch.Generator().manual_seed(seed)
    dt = R.DT[dtype]
    new, kv = [n for n, _ in lens], [l for _, l in lens]
    held = [R.ceil_div(l, page) for l in kv]
    cols, n_pages = max(held + [1]) + cols_pad, sum(held) + 2
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), cols + stride_pad), -3, dtype=torch.int32)
    cache = torch.randn(n_pages, 2, hkv, page, d, generator=g)
    cache[:, 0] *= amp
    cache = cache.to(dt)
    used = torch.zeros(n_pages, page, dtype=torch.bool)
    at = 0
    for r, h in enumerate(held):
        table[r, :h] = order[at:at + h]
        for b in range(h):
            used[int(order[at + b]), :max(0, min(page, kv[r] - b * page))] = True
        at += h
    if garbage:
        bad = (~used)[:, None, None, :, None].expand_as(cache)
        cache[bad] = float("nan")
        cache[:, 1][bad[:, 1] & (torch.rand(cache[:, 1].shape, generator=g) < 0.3)] = float("inf")
    t = sum(new)
    q = torch.randn(t, hq * d + q_pad, generator=g).to(dt)[:, :hq * d].unflatten(1, (hq, d))
    q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return q, cache, table, cols, q_start, np.asarray(kv, np.int32), max(new)


def run_attn(dtype, hq, hkv, d, page, window, lens, scale=None, seed=0, stride_pad=0, q_pad=0, pad_rows=0, amp=1.0, stream=None):
    q, cache, table, cols, q_start, kv, max_new = make_attn(dtype, hq, hkv, d, page, window, lens, seed, stride_pad=stride_pad, q_pad=q_pad, amp=amp)
    t = q.shape[0]
    scale = d ** -0.5 if scale is None else scale
    ref, lse_ref, wabs, vabs = R.attention(q, cache, table, q_start, kv, page, window, scale)
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=cache.shape[0], max_requests=len(lens),
                               max_tokens=max(t + pad_rows, 1), max_pages=cols, dtype=dtype, window=window))
    dt = R.DT[dtype]
    qd = torch.full((t + pad_rows, hq * d + q_pad), float("nan"), dtype=dt, device=DEV)
    qd[:t, :hq * d] = q.reshape(t, hq * d).to(DEV)
    qd = qd[:, :hq * d].unflatten(1, (hq, d))
    out = torch.full((t + pad_rows, hq * d + 2 * q_pad), 77.0, dtype=dt, device=DEV)
    ov = out[:, :hq * d].unflatten(1, (hq, d))
    lse = torch.full((t + pad_rows, hq), 77.0, device=DEV)
    cd, td = cache.to(DEV), table.to(DEV)[:, :cols]
    qs, kvd = i32(q_start), i32(kv)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        h.plan(qs, kvd, t + pad_rows, max_new)
        for _ in range(2):                                        # the partition serves every layer of the step
            h.forward(qd, cd, td, ov, lse=lse, scale=scale)
        h2 = ov.clone()
        h.forward(qd, cd, td, ov, scale=scale)
    torch.cuda.synchronize()
    assert h.sync_status() == 0
    assert torch.equal(h2, ov)                                    # same bits every time
    got, gl = ov[:t].double().cpu(), lse[:t].double().cpu()
    smax = float(lse_ref[torch.isfinite(lse_ref)].abs().max()) if torch.isfinite(lse_ref).any() else 0.0
    bound = R.attention_bound(dtype, ref, wabs, vabs, smax)
    assert torch.isfinite(got).all()
    err = (got - ref).abs()
    assert (err <= bound).all(), float((err / bound).max())
    empty = torch.isinf(lse_ref)
    assert (gl[empty] == -float("inf")).all() and (got[empty] == 0).all()
    # lse: float scores (2^-17 of their magnitude), exponentials and sums (2^-16 together)
    assert ((gl - lse_ref).abs()[~empty] <= 2.0 ** -15 * (1 + smax)).all()
    assert (ov[t:] == 77.0).all() and (out[:, hq * d:] == 77.0).all() and (lse[t:] == 77.0).all()
    h.destroy()


HEADS = [(32, 4, 128), (8, 8, 128), (16, 2, 64), (7, 1, 128), (12, 1, 64), (20, 4, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_attention_single_tokens(dtype, hq, hkv, d, page):
    run_attn(dtype, hq, hkv, d, page, 0, [(1, 1), (1, 2), (1, page), (1, page + 1), (1, 63), (1, 64), (1, 65), (1, 300), (1, 517)], seed=page + d)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_attention_chunks(dtype, hq, hkv, d):
    run_attn(dtype, hq, hkv, d, 32, 0, [(33, 33), (17, 150), (1, 40), (70, 200), (2, 129), (128, 128), (3, 7)], seed=d, q_pad=8, stride_pad=3)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention_page_sizes(page):
    run_attn("bf16", 8, 2, 128, page, 0, [(1, 257), (50, 300), (1, 128), (40, 40)], seed=page)
    run_attn("fp16", 4, 4, 64, page, 0, [(1, 129), (129, 300)], seed=page)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 100, 128, 1000])
def test_attention_window(window):
    run_attn("bf16", 8, 2, 128, 16, window, [(1, 1), (1, 64), (1, 333), (40, 40), (40, 400), (3, 130)], seed=window)
    run_attn("fp16", 8, 1, 64, 32, window, [(1, 200), (200, 200), (33, 700)], seed=window)


def test_attention_rows_that_see_nothing():
    """No cached token at all, and more new rows than cached tokens (the first rows stand before position 0)."""
    run_attn("bf16", 8, 2, 128, 16, 0, [(1, 0), (40, 0), (1, 5), (40, 13), (2, 1), (0, 0), (0, 50), (30, 3)])
    run_attn("fp16", 16, 2, 64, 32, 4, [(1, 0), (40, 13), (300, 7), (0, 9)])


@pytest.mark.parametrize("n_req", [1, 40, 300])
def test_attention_many_requests(n_req):
    rng = np.random.default_rng(n_req)
    lens = [(int(rng.choice([0, 1, 1, 1, 2, 5])), 0) for _ in range(n_req)]
    lens = [(max(n, 1) if i == 0 else n, n + int(rng.integers(0, 200))) for i, (n, _) in enumerate(lens)]
    run_attn("bf16", 16, 4, 64, 16, 0, lens, seed=n_req, pad_rows=9)


def test_attention_long_and_short_items_in_turn():
    """Requests with more and with fewer than 128 rows in turn, several of both in every CTA's share, some of them cut."""
    rng = np.random.default_rng(77)
    lens = []
    for i in range(60):
        n = int(rng.choice([3, 5, 9, 17, 33, 70]))
        lens.append((n, n + int(rng.integers(0, 400))))
    run_attn("bf16", 16, 2, 64, 16, 0, lens, seed=77)
    run_attn("fp16", 28, 4, 128, 32, 0, lens[:30], seed=78)
    run_attn("bf16", 16, 2, 128, 64, 150, lens[:40], seed=79)


def test_attention_one_long_request():
    """A single token and a few tokens over a long cache: the keys of one request are shared out and joined."""
    run_attn("bf16", 8, 1, 128, 64, 0, [(1, 20011)], seed=5)
    run_attn("bf16", 16, 1, 128, 64, 0, [(3, 9001)], seed=6)
    run_attn("fp16", 4, 2, 64, 16, 0, [(9, 5000), (1, 4097)], seed=7)


def test_attention_wide_groups():
    run_attn("bf16", 64, 1, 128, 16, 0, [(1, 100), (3, 77), (20, 140)], seed=8)
    run_attn("fp16", 48, 2, 64, 16, 0, [(1, 100), (5, 300)], seed=9)
    run_attn("bf16", 17, 1, 64, 16, 0, [(1, 100), (9, 9)], seed=10)


def test_attention_large_scores():
    """Scores far from zero, growing along the keys: the running maximum moves all the time."""
    run_attn("bf16", 8, 2, 128, 16, 0, [(1, 600), (60, 500)], seed=11, scale=1.0, amp=3.0)
    run_attn("fp16", 8, 2, 64, 16, 0, [(1, 600), (60, 500)], seed=12, scale=2.0)
    run_attn("bf16", 8, 2, 64, 16, 0, [(1, 300), (60, 200)], seed=13, scale=0.0)
    run_attn("bf16", 8, 2, 64, 16, 0, [(1, 300), (60, 200)], seed=14, scale=-0.3)


def test_attention_on_another_stream():
    s = torch.cuda.Stream()
    run_attn("bf16", 8, 2, 128, 16, 0, [(1, 600), (60, 500)], seed=15, stream=s)


def test_attention_of_requests_that_were_not_admitted():
    """Their rows become zeros, the others are what they are without them."""
    hq, hkv, d, page = 8, 2, 64, 16
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=8, max_requests=3, max_tokens=64, max_pages=4))
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    o = dict(q_start=z(4), kv_len=z(3), n_free_out=z(1), admitted=z(3), position=z(45), slot=z(45))
    tab, fr = torch.full((3, 4), -1, dtype=torch.int32, device=DEV), i32([3, 5, 1, 0, 0, 0, 0, 0])
    h.slots(i32([3, 40, 2]), i32([0, 0, 0]), tab, fr, i32([3]), 40, **o)
    assert o["admitted"].tolist() == [1, 0, 0] and o["n_free_out"].tolist() == [2]
    cache = torch.randn(8, 2, hkv, page, d, device=DEV).bfloat16()
    q = torch.randn(45, hq, d, device=DEV).bfloat16()
    out = torch.full((45, hq, d), 7.0, device=DEV).bfloat16()
    h.forward(q, cache, tab, out)
    assert h.sync_status() == 0
    assert (out[3:] == 0).all()
    ref, _, wabs, vabs = R.attention(q[:3].cpu(), cache.cpu(), tab.cpu(), [0, 3], [3], page, 0, d ** -0.5)
    assert ((out[:3].double().cpu() - ref).abs() <= R.attention_bound("bf16", ref, wabs, vabs, 8.0)).all()
    h.destroy()


def test_attention_bad_pages_are_latched_not_followed():
    q, cache, table, cols, q_start, kv, max_new = make_attn("bf16", 8, 2, 64, 16, 0, [(1, 100), (40, 100)])
    table[0, 2], table[1, 3] = 1 << 30, -1
    h = A.FtAttn(A.make_config(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=cache.shape[0], max_requests=2, max_tokens=64, max_pages=cols))
    h.plan(i32(q_start), i32(kv), 41, max_new)
    h.forward(q.to(DEV), cache.to(DEV), table.to(DEV), torch.empty(41, 8, 64, device=DEV).bfloat16())
    assert h.sync_status() == B.FT_ERR_INVALID_ARG and h.sync_status() == 0
    h.destroy()


def test_plan_bad_lengths_are_latched():
    h = A.FtAttn(A.make_config(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=4, max_requests=2, max_tokens=64, max_pages=4))
    for qs, kv in (([0, 3, 99], [3, 3]), ([0, 5, 4], [5, 5]), ([0, 1, 2], [1, 65]), ([0, 1, 2], [-1, 1]), ([0, 41, 42], [41, 1])):
        h.plan(i32(qs), i32(kv), 60, 40)
        assert h.sync_status() == B.FT_ERR_INVALID_ARG and h.sync_status() == 0
    h.destroy()


def test_waits_that_run_out_are_reported_and_leave_the_handle_usable():
    """A producer withholds one copy: the bounded waits give up, the kernels return, the status says so once, and the next
    calls are right again."""
    hq, hkv, d, page = 8, 2, 128, 16
    q, cache, table, cols, q_start, kv, max_new = make_attn("bf16", hq, hkv, d, page, 0, [(1, 900), (60, 300), (2, 700)], seed=21)
    ref, _, wabs, vabs = R.attention(q, cache, table, q_start, kv, page, 0, d ** -0.5)
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=cache.shape[0], max_requests=3,
                               max_tokens=6400, max_pages=cols))
    qd, cd, td = q.to(DEV), cache.to(DEV), table.to(DEV)
    x = torch.randn(6400, hq + 2 * hkv, d, device=DEV).bfloat16()
    ids = torch.arange(6400, device=DEV, dtype=torch.int32)
    rope_cache = torch.zeros_like(cd)
    many = lambda o: h.qk_rope(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], o, rope_cache, ids, torch.full_like(ids, -1))
    good = torch.empty(6400, hq, d, device=DEV).bfloat16()
    many(good)
    for mask in (1, 2, 4):
        h.debug_inject(mask, 2000)
        out, o = torch.zeros_like(qd), torch.zeros_like(good)
        if mask == 4:
            many(o)
        else:
            h.plan(i32(q_start), i32(kv), q.shape[0], max_new)
            h.forward(qd, cd, td, out)
        assert h.sync_status() == B.FT_ERR_TIMEOUT and h.sync_status() == 0
        h.debug_inject(0, 0)
        h.plan(i32(q_start), i32(kv), q.shape[0], max_new)
        h.forward(qd, cd, td, out)
        many(o)
        assert h.sync_status() == 0 and torch.equal(o, good)
        assert ((out.double().cpu() - ref).abs() <= R.attention_bound("bf16", ref, wabs, vabs, 12.0)).all()
    h.destroy()


def test_refusals():
    h = A.FtAttn(A.make_config(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=4, max_requests=2, max_tokens=8, max_pages=4))
    q, out = (torch.zeros(2, 8, 64, device=DEV).bfloat16() for _ in range(2))
    cache, tab = torch.zeros(4, 2, 2, 16, 64, device=DEV).bfloat16(), i32(np.zeros((2, 4)))

    def refuses(code, f, *a, **k):
        with pytest.raises(B.FtMoeError) as e:
            f(*a, **k)
        assert e.value.code == code

    bad = B.FT_ERR_INVALID_ARG
    refuses(B.FT_ERR_STATE, h.forward, q, cache, tab, out)
    refuses(bad, h.plan, i32([0, 1, 2]), i32([1, 1]), 9, 1)                                # more rows than max_tokens
    refuses(bad, h.plan, i32([0, 1, 2, 3]), i32([1, 1, 1]), 3, 1)                          # more requests than max_requests
    refuses(bad, h.plan, i32([0, 1]), i32([1, 1]), 2, 1)                                   # q_start too short
    refuses(bad, h.plan, i32([0, 1, 2]).long(), i32([1, 1]), 2, 1)
    h.plan(i32([0, 1, 2]), i32([1, 1]), 2, 1)
    refuses(bad, h.forward, q.half(), cache, tab, out)
    refuses(bad, h.forward, q[:1], cache, tab, out)
    refuses(bad, h.forward, q.cpu(), cache, tab, out)
    refuses(bad, h.forward, q, cache[:3], tab, out)
    refuses(bad, h.forward, q, cache, tab[:, :3], out)
    refuses(bad, h.forward, q, cache, tab.float(), out)
    refuses(bad, h.forward, q, cache, tab, out, scale=float("nan"))
    refuses(bad, h.forward, torch.zeros(2, 64, 8, device=DEV).bfloat16().transpose(1, 2), cache, tab, out)
    odd = torch.zeros(2 * 8 * 64 + 4, device=DEV).bfloat16()
    refuses(bad, h.forward, odd[4:].view(2, 8, 64), cache, tab, out)                       # 8-byte aligned only
    refuses(bad, h.forward, torch.zeros(2, 8 * 64 + 4, device=DEV).bfloat16()[:, :512].unflatten(1, (8, 64)), cache, tab, out)
    p, s = i32([0, 0]), i32([0, 1])
    kv = torch.zeros(2, 2, 64, device=DEV).bfloat16()
    cs = torch.zeros(4, 64, device=DEV)
    refuses(bad, h.qk_rope, q, kv, kv, out, cache, p[:1], s, cs)
    refuses(bad, h.qk_rope, q, kv[:1], kv, out, cache, p, s, cs)
    refuses(bad, h.qk_rope, q, kv, kv, out, cache, p, s, torch.zeros(4, 72, device=DEV))   # wider than the head
    refuses(bad, h.qk_rope, q, kv, kv, out, cache, p, s, torch.zeros(4, 20, device=DEV))   # not a multiple of 8
    refuses(bad, h.qk_rope, q, kv, kv, out, cache, p, s, cs.double())
    refuses(bad, h.qk_rope, q, kv, kv, out, cache, p, s, cs, w_q=torch.ones(32, device=DEV).bfloat16())
    refuses(bad, h.qk_rope, q, kv, kv, out, cache, p, s, cs, eps=float("nan"))
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    o = dict(q_start=z(3), kv_len=z(2), n_free_out=z(1), admitted=z(2), position=z(2), slot=z(2))
    refuses(bad, h.slots, z(2), z(2), tab, z(3), z(1), 1, **o)                             # free_pages shorter than the pool
    f = z(1)
    refuses(bad, h.slots, z(2), z(2), tab, z(4), f, 1, **{**o, "n_free_out": f})           # counts in place
    refuses(bad, h.slots, z(2), z(2), tab, z(4), f, 3, **o)                                # max_new > rows
    refuses(bad, h.slots, z(2), z(2), tab, z(4), f, 1, **{**o, "slot": z(1)})
    assert h.sync_status() == 0
    h.destroy()
