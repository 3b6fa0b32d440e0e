"""The dense operators as they are used: a served decoder with 4-bit weights (every call checked against its 64-bit form), a chain of them in
a captured graph, calls of one handle at the same time, other streams, waits that give up."""
import numpy as np
import pytest
import torch

from examples import serve_decoder as S
from paper_2608_16157_b200 import binding as B
from paper_2608_16157_b200 import dense as D
from tests import dense_reference as R
from tests.test_gpu_dense import DEV, gen, make_w4

pytestmark = pytest.mark.gpu


def test_a_served_decoder_with_4_bit_weights():
    rng = np.random.default_rng(5)
    dec = S.Decoder(layers=2, n_pages=12, max_requests=4, max_tokens=64, max_pages=8, seed=5, w4=True)
    prompts = [rng.integers(0, dec.vocab, n).tolist() for n in (60, 1, 33, 50)]
    mats = {id(w): R.w4_weights(*S.quantise(m), None) for w, m in zip(dec.w4_qkv + dec.w4_o + [dec.w4_head], dec.w_qkv + dec.w_o + [dec.head])}
    h, calls = dec.dense, {"norm": 0, "w4": 0, "logp": 0}
    add_norm, w4, logprobs = h.add_norm, h.w4, h.logprobs

    def near(got, ref, tol):
        assert ((got.double() - ref).abs() <= tol + R.rounding(ref, got.dtype)).all()

    def checked_norm(y, res, res_out, out, **kw):
        ref = R.add_norm(y, res, None, None, None, post=False, w_offset=0.0, eps=kw["eps"], res_scale=1.0, y_scale=1.0)
        add_norm(y, res, res_out, out, **kw)
        if res_out is not None:
            near(res_out, ref[0], ref[2])
        near(out, ref[1], ref[3])
        calls["norm"] += 1

    def checked_w4(x, weight, y, **kw):
        ref, tol = R.w4(x, mats[id(weight)], None, y.dtype)
        w4(x, weight, y, **kw)
        near(y, ref, tol)
        calls["w4"] += 1

    def checked_logprobs(logits, *, entropy, top_ids, top_logprobs):
        logp, ent, ids, tol, tol_ent = R.logprobs(logits, 1.0, top_ids.shape[1])
        logprobs(logits, entropy=entropy, top_ids=top_ids, top_logprobs=top_logprobs)
        assert torch.equal(top_ids.long(), ids)
        near(top_logprobs, logp.gather(1, ids), tol.gather(1, ids))
        near(entropy, ent, tol_ent)
        calls["logp"] += 1

    h.add_norm, h.w4, h.logprobs = checked_norm, checked_w4, checked_logprobs
    answers = S.serve(dec, prompts, n_new=5, chunk=24)
    assert all(len(a) == 5 and all(0 <= t < dec.vocab for t in a) for a in answers)
    assert h.sync_status() == 0 and dec.attn.sync_status() == 0 and dec.moe.sync_status() == 0 and int(dec.n_free) == 12
    assert min(calls.values()) >= 5 and calls["norm"] == 5 * calls["logp"] and calls["w4"] == 5 * calls["logp"]
    del h.add_norm, h.w4, h.logprobs
    dec.close()


def chain(h, x, res, mats, head, logits, buf):
    """norm -> wide projection -> narrow projection -> residual + norm -> head -> log probabilities."""
    h.add_norm(None, res, None, buf["h"])
    h.w4(buf["h"], mats[0], buf["wide"])
    h.w4(buf["wide"], mats[1], buf["y"])
    h.add_norm(buf["y"], res, buf["res"], buf["h"], post=True, y_scale=0.5)
    h.w4(buf["h"], head, logits)
    h.logprobs(logits, entropy=buf["entropy"], top_ids=buf["ids"], top_logprobs=buf["top"])


def make_chain(h, t, seed):
    d, wide, vocab = 512, 1280, 3001
    mats = [h.w4_pack(*make_w4(wide, d, 128, "bf16", True, seed)), h.w4_pack(*make_w4(d, wide, 64, "bf16", False, seed + 1))]
    head = h.w4_pack(*make_w4(vocab, d, 32, "bf16", False, seed + 2)[:2])
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device=DEV)
    buf = dict(h=z(t, d), wide=z(t, wide), y=z(t, d), res=z(t, d), entropy=z(t, dt=torch.float32), ids=z(t, 4, dt=torch.int32), top=z(t, 4, dt=torch.float32))
    res = torch.randn(t, d, generator=gen(seed), device=DEV).bfloat16()
    return res, mats, head, z(t, vocab, dt=torch.float32), buf


@pytest.mark.parametrize("t", [1, 7, 20, 100, 300])
def test_a_chain_replayed_from_a_graph(t):
    """Every result of a replay on new inputs is bit for bit that of the calls one by one."""
    h = D.FtDense()
    res, mats, head, logits, buf = make_chain(h, t, t)
    chain(h, None, res, mats, head, logits, buf)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            chain(h, None, res, mats, head, logits, buf)
        for i in range(3):
            res.copy_(torch.randn(res.shape, generator=gen(50 + i), device=DEV))
            chain(h, None, res, mats, head, logits, buf)
            want = {k: v.clone() for k, v in buf.items()}
            for v in buf.values():
                v.zero_()
            g.replay()
            st.synchronize()
            for k, v in buf.items():
                assert torch.equal(v, want[k]), k
    assert h.sync_status() == 0
    h.destroy()


def test_calls_of_one_handle_at_the_same_time():
    """The kernels share no workspace: chains on four streams, from graphs and eager, in any overlap."""
    h = D.FtDense()
    sets = [make_chain(h, t, t) for t in (3, 40, 130, 1)]
    want = []
    for s in sets:
        chain(h, None, *s)
        want.append({k: v.clone() for k, v in s[-1].items()})
    torch.cuda.synchronize()
    streams, graphs = [torch.cuda.Stream() for _ in sets], []
    for s, st in zip(sets, streams):
        with torch.cuda.stream(st):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                chain(h, None, *s)
            graphs.append(g)
    for i in range(20):
        for s, st, g in zip(sets, streams, graphs):
            with torch.cuda.stream(st):
                g.replay() if i % 3 else chain(h, None, *s)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        for k, v in s[-1].items():
            assert torch.equal(v, w[k]), k
    assert h.sync_status() == 0
    h.destroy()


def test_results_do_not_change_from_call_to_call():
    h = D.FtDense()
    for t, n, k in ((1, 2048, 4096), (8, 5120, 2048), (30, 2048, 2048), (64, 1024, 7168), (200, 700, 4096)):
        w = h.w4_pack(*make_w4(n, k, 128, "fp16", True, 3))
        x = torch.randn(t, k, generator=gen(4), device=DEV).half()
        for dt in (torch.float16, torch.float32):
            a, b = torch.empty(t, n, dtype=dt, device=DEV), torch.empty(t, n, dtype=dt, device=DEV)
            h.w4(x, w, a)
            for _ in range(10):
                b.fill_(float("nan"))
                h.w4(x, w, b)
                assert torch.equal(a, b)
    h.destroy()


def test_inputs_made_on_another_stream_and_an_explicit_stream():
    h = D.FtDense()
    st = torch.cuda.Stream()
    x = torch.empty(9, 256, dtype=torch.bfloat16, device=DEV)
    out, y = torch.empty_like(x), torch.empty(9, 48, device=DEV)
    w = h.w4_pack(*make_w4(48, 256, 64, "bf16", False, 1))
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(20_000_000)
        x.fill_(2.0)
        h.add_norm(None, x, None, out)              # the current stream
    h.w4(out, w, y, stream=st)                      # a stream object
    h.w4(out, w, y, stream=st.cuda_stream)          # its handle
    st.synchronize()
    assert (out == 1).all()
    assert torch.allclose(y[0].double(), R.w4_weights(*make_w4(48, 256, 64, "bf16", False, 1)).sum(1), atol=1e-4)
    h.destroy()


@pytest.mark.parametrize("t,out32,mask", [(2, False, 1), (12, True, 1), (30, True, 1), (40, False, 2), (200, False, 2), (70, True, 2)])
@pytest.mark.parametrize("n,k", [(300, 512), (2048, 4096)])
def test_waits_that_give_up(t, out32, mask, n, k):
    """A copy that never comes: the call ends, the status says so once, and the handle works on."""
    h = D.FtDense()
    codes, scales, _ = make_w4(n, k, 128, "bf16", False, 1)
    w = h.w4_pack(codes, scales)
    x = torch.randn(t, k, generator=gen(2), device=DEV).bfloat16()
    y = torch.empty(t, n, dtype=torch.float32 if out32 else torch.bfloat16, device=DEV)
    try:
        h.debug_inject(mask, 2000)
        h.w4(x, w, y)
        assert h.sync_status() == B.FT_ERR_TIMEOUT and h.sync_status() == 0
    finally:
        h.debug_inject(0, 0)
    h.w4(x, w, y)
    assert h.sync_status() == 0
    ref, tol = R.w4(x, R.w4_weights(codes, scales, None), None, y.dtype)
    assert ((y.double() - ref).abs() <= tol + R.rounding(ref, y.dtype)).all()
    h.destroy()


def test_images_and_logits_beyond_32_bit_offsets():
    """A matrix whose image and results, and logits whose rows, stand more than 2^32 bytes from their start."""
    h = D.FtDense()
    n, k = 1 << 21, 4352                              # 4.7 GB of records
    size = D.w4_bytes(n, k, 128)
    assert size > 1 << 32
    codes = torch.randint(0, 256, (n, k // 2), generator=gen(1), device=DEV, dtype=torch.uint8)
    scales = torch.full((n, k // 128), 0.01, device=DEV).bfloat16()
    w = h.w4_pack(codes, scales)
    for t in (2, 40):
        x = torch.randn(t, k, generator=gen(2), device=DEV).bfloat16()
        y = torch.empty(t, n, device=DEV, dtype=torch.bfloat16)
        h.w4(x, w, y)
        rows = torch.cat([torch.arange(200), torch.arange(n - 200, n)]).to(DEV)
        ref, tol = R.w4(x, R.w4_weights(codes[rows], scales[rows], None), None, y.dtype)
        assert ((y[:, rows].double() - ref).abs() <= tol + R.rounding(ref, y.dtype)).all()
    del codes, w, y
    torch.cuda.empty_cache()
    rows, v = 40, 120_000_000
    logits = torch.zeros(rows, v, dtype=torch.bfloat16, device=DEV)       # 9.6 GB
    logits[:, 7] = 30.0
    logits[:, v - 3] = 31.0
    ids, top = torch.empty(rows, 2, dtype=torch.int32, device=DEV), torch.empty(rows, 2, device=DEV)
    h.logprobs(logits, top_ids=ids, top_logprobs=top)
    assert (ids[:, 0] == v - 3).all() and (ids[:, 1] == 7).all()
    lse = np.log(np.exp(30.0) + np.exp(31.0) + v - 2)
    assert (top.double() - torch.tensor([31 - lse, 30 - lse], device=DEV)).abs().max() < 1e-4
    assert h.sync_status() == 0
    h.destroy()
