"""GPU tests of the attention operators at their edges: windows, infinities and NaN, entries that cannot be, empty steps, long
prompts, many work items, replay from a graph."""
import numpy as np
import pytest
import torch

from paper_2608_16157_b200 import attention as A
from paper_2608_16157_b200 import binding as B
from tests import attn_reference as R
from tests.test_gpu_attn import DEV, i32, make_attn, run_attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 30, 1 << 30])
def test_a_window_wider_than_any_request_is_no_window(window):
    """Also for requests whose first rows stand before position 0 (more new rows than cached tokens)."""
    run_attn("bf16", 8, 2, 128, 16, window, [(1, 0), (40, 13), (2, 1), (30, 3), (60, 300), (1, 70)], seed=1)
    run_attn("fp16", 16, 2, 64, 32, window, [(40, 13), (300, 7), (0, 9), (2, 100)], seed=2)


@pytest.mark.parametrize("d,rot,inter,norm,pad", [(128, 64, False, False, 0), (128, 64, False, True, 4), (64, 0, False, False, 0), (64, 32, True, False, 4),
                                                  (128, 16, True, True, 0), (64, 24, False, False, 0)])
@pytest.mark.parametrize("t", [5, 9001])
def test_qk_rope_infinities_stay_in_their_element(d, rot, inter, norm, pad, t):
    """An infinity or a NaN outside the rotated part reaches no other element: without a norm what is not rotated is copied; with
    one (infinite mean square) every other finite element becomes 0."""
    hq, hkv, page = 6, 2, 16
    n_pages = R.ceil_div(t, page)
    g = torch.Generator().manual_seed(d + rot)
    x = torch.randn(t, (hq + 2 * hkv) * d + pad, generator=g).bfloat16()
    view = x[:, :(hq + 2 * hkv) * d].unflatten(1, (hq + 2 * hkv, d))
    bad = [rot + i for i in (0, 1, (d - rot) // 2, (d - rot) // 2 + 3, d - rot - 1)]
    for i, b in enumerate(bad):
        view[i % t, i % (hq + hkv), b] = [float("inf"), -float("inf"), float("nan")][i % 3]
    cs = torch.randn(t, rot, generator=g).to(DEV) if rot else None
    w = (1 + 0.3 * torch.randn(d, generator=g)).bfloat16().to(DEV) if norm else None
    ids = torch.arange(t, dtype=torch.int32, device=DEV)
    xd = x.to(DEV)[:, :(hq + 2 * hkv) * d].unflatten(1, (hq + 2 * hkv, d))
    out, cache = torch.zeros(t, hq, d, device=DEV).bfloat16(), torch.zeros(n_pages, 2, hkv, page, d, device=DEV).bfloat16()
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=n_pages, max_requests=1, max_tokens=t, max_pages=4))
    h.qk_rope(xd[:, :hq], xd[:, hq:hq + hkv], xd[:, hq + hkv:], out, cache, ids, ids, cs, w_q=w, w_k=w)
    assert h.sync_status() == 0
    keys = cache[:, 0].permute(0, 2, 1, 3).reshape(n_pages * page, hkv, d)[:t]
    got, src = torch.cat([out, keys], 1).cpu(), view[:, :hq + hkv]
    if not norm:
        assert torch.equal(torch.nan_to_num(got[..., rot:], 9e9, 8e9, 7e9), torch.nan_to_num(src[..., rot:], 9e9, 8e9, 7e9))
        assert torch.isfinite(got[..., :rot]).all()
    else:
        hit = ~torch.isfinite(src.float()).all(-1)                    # heads with an infinity or a NaN
        assert torch.isfinite(got[~hit].float()).all() and hit.sum() == min(len(bad), t)
        inf = torch.isinf(src.float()).any(-1)
        assert torch.equal(torch.isnan(got[inf]), torch.isinf(src[inf])) and (torch.nan_to_num(got[inf].float()) == 0).all()
    h.destroy()


@pytest.mark.parametrize("d", [64, 128])
def test_lse_of_rows_with_infinite_or_nan_scores(d):
    """Such a row is no row that attends to nothing: its result and its lse are NaN, those of the others do not change."""
    hq, hkv, page = 8, 2, 16
    lens = [(1, 70), (1, 900), (40, 300), (200, 700), (1, 33), (50, 60)]
    q, cache, table, cols, q_start, kv, max_new = make_attn("bf16", hq, hkv, d, page, 0, lens, seed=3)
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=cache.shape[0], max_requests=len(lens),
                               max_tokens=q.shape[0], max_pages=cols))
    h.plan(i32(q_start), i32(kv), q.shape[0], max_new)
    q[int(q_start[1]), :, 0] = 1.0                    # (its score with the infinite key is +infinity)
    res = []
    for bad in (False, True):
        if bad:        # kv head 1, the first element of one key of the first four requests
            for r, (j, v) in enumerate(((5, "nan"), (640, "inf"), (7, "nan"), (130, "nan"))):
                cache[int(table[r, j // page]), 0, 1, j % page, 0] = float(v)
        out, lse = torch.zeros_like(q, device=DEV).contiguous(), torch.zeros(q.shape[0], hq, device=DEV)
        h.forward(q.to(DEV), cache.to(DEV), table.to(DEV)[:, :cols], out, lse=lse)
        assert h.sync_status() == 0
        res.append((out.cpu(), lse.cpu()))
    (o0, l0), (o1, l1) = res
    assert torch.isfinite(l0).all()
    nan = torch.zeros_like(l0, dtype=torch.bool)
    nan[:int(q_start[4]), hq // 2:] = True          # (every row of these requests attends to the key in question)
    assert torch.isnan(l1[nan]).all() and torch.isnan(o1[nan]).all()
    assert torch.equal(l1[~nan], l0[~nan]) and torch.equal(o1[~nan], o0[~nan])
    h.destroy()


@pytest.mark.parametrize("dtype,hq,hkv,d,page", [("bf16", 8, 2, 64, 16), ("fp16", 16, 2, 128, 32), ("bf16", 8, 1, 128, 128), ("fp16", 4, 4, 64, 64)])
def test_attention_of_a_bad_page_reads_no_other_page(dtype, hq, hkv, d, page):
    """A page id outside the pool stands for a page of zeros: results do not depend on what any other request's pages hold, and the
    requests with good tables are what they were."""
    lens = [(1, 500), (60, 700), (1, 400), (60, 500), (1, 4 * page), (40, 4 * page)]
    q, cache, table, cols, q_start, kv, max_new = make_attn(dtype, hq, hkv, d, page, 0, lens, seed=4)
    owner = {int(p): r for r in range(len(lens)) for p in table[r, :R.ceil_div(lens[r][1], page)]}
    zero = min(p for p in range(cache.shape[0]) if p not in owner)          # a page of nobody, for the reference
    zeros = table.clone()
    cache[zero] = 0
    for r, b, p in ((0, 2, cache.shape[0]), (1, 1, -1), (1, 3, 1 << 30), (4, 0, -(1 << 31))):
        table[r, b], zeros[r, b] = p, zero
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=cache.shape[0], max_requests=len(lens),
                               max_tokens=q.shape[0], max_pages=cols, dtype=dtype))
    ref, lse_ref, wabs, vabs = R.attention(q, cache, zeros, q_start, kv, page, 0, d ** -0.5)
    bound = R.attention_bound(dtype, ref, wabs, vabs, float(lse_ref.abs().max()))
    poison = cache.clone()
    for p in range(cache.shape[0]):                              # every page that is not of the requests with bad entries
        if owner.get(p) not in (0, 1, 4):
            poison[p] = float("nan")
    for c, rows in ((cache, range(len(lens))), (poison, (0, 1, 4))):
        h.plan(i32(q_start), i32(kv), q.shape[0], max_new)
        out = torch.zeros(q.shape, dtype=q.dtype, device=DEV)
        h.forward(q.to(DEV), c.to(DEV), table.to(DEV), out)
        assert h.sync_status() == B.FT_ERR_INVALID_ARG and h.sync_status() == 0
        for r in rows:
            z = slice(int(q_start[r]), int(q_start[r + 1]))
            assert ((out[z].double().cpu() - ref[z]).abs() <= bound[z]).all(), r
    h.destroy()


@pytest.mark.parametrize("chunk", [1, 40])
def test_steps_replayed_from_a_graph(chunk):
    """slots, qk_rope and forward captured once; every replay takes the lengths, tables and activations that are there then."""
    hq, hkv, d, page, n_pages, n_req, cols = 8, 2, 128, 16, 200, 6, 40
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=n_pages, max_requests=n_req,
                               max_tokens=n_req * chunk, max_pages=cols))
    t = n_req * chunk
    rng, g = np.random.default_rng(chunk), torch.Generator().manual_seed(chunk)
    z = lambda *n: torch.zeros(*n, dtype=torch.int32, device=DEV)
    new, ctx, tab, fr, nf = z(n_req), z(n_req), z(n_req, cols), i32(rng.permutation(n_pages)), i32([n_pages])
    o = dict(q_start=z(n_req + 1), kv_len=z(n_req), n_free_out=z(1), admitted=z(n_req), position=z(t), slot=z(t))
    x, cs = torch.zeros(t, hq + 2 * hkv, d, device=DEV).bfloat16(), torch.randn(cols * page, d, generator=g).to(DEV)
    q, out = (torch.zeros(t, hq, d, device=DEV).bfloat16() for _ in range(2))
    cache = torch.zeros(n_pages, 2, hkv, page, d, device=DEV).bfloat16()

    def step():
        h.slots(new, ctx, tab, fr, nf, chunk, **o)
        for _ in range(2):                                     # two layers (of one cache)
            h.qk_rope(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, cache, o["position"], o["slot"], cs)
            h.forward(q, cache, tab, out)

    state = [tab, fr, cache, q, out, *o.values()]
    first = [s.clone() for s in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                 # (nothing to do yet: all lengths are 0)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for s, f in zip(state, first):
        s.copy_(f)
    for i in range(12):
        lens = [int(rng.integers(0, chunk + 1)) if rng.random() < 0.8 else chunk for _ in range(n_req)]
        if i == 7:
            lens[2] = -1
        new.copy_(i32(lens))
        x.copy_(torch.randn(x.shape, generator=g).bfloat16())
        before = [s.clone() for s in state]
        graph.replay()
        assert h.sync_status() == 0
        replayed = [s.clone() for s in state]
        for s, b in zip(state, before):
            s.copy_(b)
        step()                                                 # the same step by calls: the same bits
        assert h.sync_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(state, replayed))
        assert o["admitted"].tolist() == [int(n >= 0) for n in lens]
        rows = int(o["q_start"][-1])
        ref, _, wabs, vabs = R.attention(q[:rows].cpu(), cache.cpu(), tab.cpu(), o["q_start"].tolist(), o["kv_len"].tolist(), page, 0, d ** -0.5)
        assert ((out[:rows].double().cpu() - ref).abs() <= R.attention_bound("bf16", ref, wabs, vabs, 60.0)).all()
        ctx.copy_(o["kv_len"])
        nf.copy_(o["n_free_out"])
    del graph
    h.destroy()


@pytest.mark.parametrize("t", [0, 3])
def test_a_step_without_requests(t):
    h = A.FtAttn(A.make_config(n_q_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=6, max_requests=4, max_tokens=8, max_pages=4))
    z = lambda n: torch.full((n,), 9, dtype=torch.int32, device=DEV)
    fr = i32([4, 2, 0, 1, 3, 5])
    for tab in (torch.zeros(0, 4, dtype=torch.int32, device=DEV), torch.zeros(2, 4, dtype=torch.int32, device=DEV)):
        o = dict(q_start=z(1), kv_len=z(0), n_free_out=z(1), admitted=z(0), position=z(t), slot=z(t))
        h.slots(z(0), z(0), tab, fr, i32([5]), 0, **o)
        assert h.sync_status() == 0
        assert o["q_start"].tolist() == [0] and o["n_free_out"].tolist() == [5] and fr.tolist() == [4, 2, 0, 1, 3, 5]
        assert o["position"].tolist() == [-1] * t and o["slot"].tolist() == [-1] * t
        q, out = torch.zeros(t, 8, 64, device=DEV).bfloat16(), torch.full((t, 8, 64), 7.0, device=DEV).bfloat16()
        h.forward(q, torch.zeros(6, 2, 2, 16, 64, device=DEV).bfloat16(), tab, out)
        assert h.sync_status() == 0 and (out == 7.0).all()
    h.slots(z(0), z(0), tab, fr, i32([7]), 0, **o)            # more free pages than there are
    assert h.sync_status() == B.FT_ERR_INVALID_ARG
    h.plan(z(1), z(0), t, 0)
    assert h.sync_status() == 0
    h.destroy()


def test_released_pages_are_counted_beyond_32_bits():
    """1024 finished requests that claim 2^22 + 1 pages each: more than the pool has, whatever the sum is modulo 2^32."""
    cols = (1 << 22) + 1
    h = A.FtAttn(A.make_config(n_q_heads=1, n_kv_heads=1, head_dim=64, page_tokens=16, n_pages=4096, max_requests=1024, max_tokens=8, max_pages=cols))
    tab = torch.empty(1024, cols, dtype=torch.int32, device=DEV)
    fr = torch.arange(4096, dtype=torch.int32, device=DEV)
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    o = dict(q_start=z(1025), kv_len=z(1024), n_free_out=z(1), admitted=z(1024), position=z(8), slot=z(8))
    h.slots(torch.full((1024,), -1, dtype=torch.int32, device=DEV), torch.full((1024,), cols * 16, dtype=torch.int32, device=DEV), tab, fr, i32([64]), 0, **o)
    assert h.sync_status() == B.FT_ERR_INVALID_ARG
    assert o["n_free_out"].tolist() == [64] and torch.equal(fr.cpu(), torch.arange(4096, dtype=torch.int32))
    h.destroy()


def tile_runs(lens, group, n_kv, window, grid):
    """Longest run of steps of the tiled kernel in which both tiles use every half of two successive blocks, from the work
    partition (items of two tiles of 128 // group tokens, blocks of 128 keys, three units an item besides its blocks)."""
    tokens = 128 // group
    entries, unit = [], 0
    for n, kv in lens:
        if n * group <= 16:
            continue
        for first in range(0, n, 2 * tokens):
            m, pos0 = min(2 * tokens, n - first), kv - n + first
            hi = max(0, pos0 + m)
            lo = min(hi, max(0, pos0 - window + 1)) if window else 0
            nb = max(1, R.ceil_div(hi, 128) - lo // 128)
            entries.append((m, pos0, lo // 128, nb, unit))
            unit += nb + 3
    quota = max(1, R.ceil_div(unit * n_kv, grid))
    best = 0
    for m, pos0, b0, nb, unit0 in entries:
        if m <= tokens:
            continue
        spans = []
        for t in range(2):
            n = min(tokens, m - t * tokens)
            hi, lo = pos0 + t * tokens + n, max(0, pos0 + t * tokens - window + 1) if window else 0
            spans.append((lo // 64, R.ceil_div(max(0, hi), 64)))
        for head in range(n_kv):
            u = unit0 * n_kv + head * (nb + 3) + 3
            for c in range(u // quota, (u + nb - 1) // quota + 1):
                k0, k1 = b0 + max(0, c * quota - u), b0 + min(nb, (c + 1) * quota - u)
                h0, h1 = max(max(2 * k0, s[0]) for s in spans), min(min(2 * k1, s[1]) for s in spans)
                best = max(best, min(k1 - k0, (h1 >> 1) - k0) - max(1, ((h0 + 2) >> 1) + 1 - k0))
    return best


def check_rows(dtype, hq, hkv, d, page, window, lens, rows, shape_keys=None, seed=0):
    """Attention of whole requests, checked at `rows` packed rows against the 64-bit form (each as a request of one token)."""
    q, cache, table, cols, q_start, kv, max_new = make_attn(dtype, hq, hkv, d, page, window, lens, seed=seed)
    if shape_keys:
        shape_keys(q, cache, table, kv)
    t = q.shape[0]
    h = A.FtAttn(A.make_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_tokens=page, n_pages=cache.shape[0], max_requests=len(lens),
                               max_tokens=t, max_pages=cols, dtype=dtype, window=window))
    out, lse = torch.full((t, hq, d), 77.0, dtype=q.dtype, device=DEV), torch.full((t, hq), 77.0, device=DEV)
    qd, cd, td = q.to(DEV), cache.to(DEV), table.to(DEV)
    h.plan(i32(q_start), i32(kv), t, max_new)
    h.forward(qd, cd, td, out, lse=lse)
    again = out.clone()
    h.forward(qd, cd, td, out)
    assert h.sync_status() == 0 and torch.equal(again, out) and torch.isfinite(out).all() and torch.isfinite(lse).all()
    req = np.searchsorted(q_start, rows, side="right") - 1
    pos = [int(kv[r]) - int(q_start[r + 1]) + int(i) for r, i in zip(req, rows)]
    ref, lse_ref, wabs, vabs = R.attention(q[rows], cache, table[req], list(range(len(rows) + 1)), [p + 1 for p in pos], page, window, d ** -0.5)
    smax = float(lse_ref.abs().max())
    err, bound = (out[rows].double().cpu() - ref).abs(), R.attention_bound(dtype, ref, wabs, vabs, smax)
    assert (err <= bound).all(), float((err / bound).max())
    assert ((lse[rows].double().cpu() - lse_ref).abs() <= 2.0 ** -15 * (1 + smax)).all()
    h.destroy()


def sample(rng, t, n):
    return np.unique(np.concatenate([[0, 1, 127, 128, t // 2, t - 129, t - 2, t - 1], rng.integers(0, t, n)]))


@pytest.mark.parametrize("dtype,hq,hkv,d,page,window,lens", [
    ("bf16", 32, 4, 128, 64, 0, [(4100, 4100)]), ("fp16", 32, 4, 128, 16, 0, [(2100, 6007)]),
    ("bf16", 64, 8, 64, 32, 0, [(3001, 4100)]), ("fp16", 10, 10, 64, 128, 0, [(5000, 5000)]),
    ("bf16", 16, 4, 128, 32, 1500, [(3000, 5000), (1, 900)]), ("fp16", 64, 8, 64, 16, 2049, [(2500, 6001)])])
def test_attention_of_long_prompts(dtype, hq, hkv, d, page, window, lens):
    """Shares of many blocks: the issuing warp's steady state runs for many steps, its ring and its parities wrap."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert tile_runs(lens, hq // hkv, hkv, window, sms) >= 8
    check_rows(dtype, hq, hkv, d, page, window, lens, sample(np.random.default_rng(d + page), lens[0][0], 56), seed=page)


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 4, 128), ("fp16", 16, 2, 64)])
def test_attention_of_a_long_prompt_with_growing_scores(dtype, hq, hkv, d):
    """The score of a key grows with its position, by more than the 2^8 that a reference allows from block to block: results are
    rescaled in every block."""
    page, n = 32, 4000

    def grow(q, cache, table, kv):
        u = torch.randn(d, generator=torch.Generator().manual_seed(5))
        u /= u.norm()
        j = torch.arange(n)
        k = cache[table[0].long()[j // page], 0, :, j % page].float() * 0.5 + (0.1 * d ** 0.5 / 4) * j[:, None, None] * u
        cache[table[0].long()[j // page], 0, :, j % page] = k.to(cache.dtype)
        q.copy_((q.float() * 0.25 + 4 * u).to(q.dtype))

    check_rows(dtype, hq, hkv, d, page, 0, [(n, n)], sample(np.random.default_rng(7), n, 40), shape_keys=grow, seed=9)


def test_attention_of_many_work_items():
    """Work lists longer than a block of the partition has threads, and longer than the positions it keeps in shared memory."""
    rng = np.random.default_rng(8)
    lens = [(int(rng.integers(5, 12)), 0) for _ in range(250)]
    lens = [(n, n + int(rng.integers(0, 60))) for n, _ in lens]
    assert 256 < sum(R.ceil_div(n, 4) for n, _ in lens) < 2048
    run_attn("bf16", 64, 1, 64, 16, 0, lens, seed=1)
    lens = [(n, kv) for n, kv in lens for _ in range(4)]
    assert sum(R.ceil_div(n, 4) for n, _ in lens) > 2048 and len(lens) <= 1024
    run_attn("fp16", 64, 1, 64, 32, 0, lens, seed=2)


def test_attention_of_a_prompt_of_many_work_items():
    check_rows("bf16", 64, 1, 64, 64, 0, [(8400, 8400)], sample(np.random.default_rng(3), 8400, 40), seed=6)
