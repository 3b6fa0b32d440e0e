"""GPU tests of the operators of ``dense`` against 64-bit forms, at the sizes, layouts and values where they can go wrong."""
import pytest
import torch

from paper_2608_16157_b200 import binding as B
from paper_2608_16157_b200 import dense as D
from tests import dense_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def wide(t, d, pad, dtype, g, shift=0, fill=NAN, scale=1.0):
    """Random [t, d] rows inside a buffer whose other elements are `fill`; returns (view, buffer)."""
    buf = torch.full((t * (d + pad) + shift + 1,), fill, dtype=dtype, device=DEV)
    v = buf[shift:shift + t * (d + pad)].view(t, d + pad)[:, :d]
    v.copy_(torch.randn(t, d, generator=g, device=DEV) * scale)
    return v, buf


def same_outside(view, buf, before):
    """Nothing but the view's elements has changed."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    view_mask = torch.as_strided(mask, view.shape, view.stride(), view.storage_offset())
    view_mask.fill_(False)
    a, b = buf[mask], before[mask]
    assert torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0))


# ------------------------------------------------------------------------------------------------------------ norm
def run_norm(t, d, dtype, res_dtype, *, post=False, gate="none", wp=True, wn=True, pad=0, shift=0, offset=0.0, eps=1e-6, has_y=True, has_res=True,
             has_res_out=True, has_out=True, inplace=False, seed=0):
    g, dt, rt = gen(seed), R.DT[dtype], R.DT[res_dtype]
    h = D.FtDense()
    y = wide(t, d, pad, dt, g, shift)[0] if has_y else None
    res = wide(t, d, pad, rt, g, shift, scale=3.0)[0] if has_res else None
    gt = {"none": None, "element": (t, d), "channel": (1, d), "token": (t, 1), "one": (1, 1)}[gate]
    gt = None if gt is None else torch.randn(*gt, generator=g, device=DEV).to(dt)
    w_post = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt) if wp and post else None
    w_pre = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt) if wn else None
    ref = R.add_norm(y, res, gt, w_post, w_pre, post=post, w_offset=offset, eps=eps, res_scale=0.9, y_scale=0.7)
    ro, ro_buf = (res, None) if inplace and has_res else wide(t, d, pad, rt, g, shift)
    out, out_buf = (y, None) if inplace and has_y else wide(t, d, pad, dt, g, shift)
    before = [None if b is None else b.clone() for b in (ro_buf, out_buf)]
    h.add_norm(y, res, ro if has_res_out else None, out if has_out else None, post=post, w_post=w_post, w_pre=w_pre, gate=gt, w_offset=offset, eps=eps,
               res_scale=0.9, y_scale=0.7)
    assert h.sync_status() == 0 and h.launch_count() == 1
    if has_res_out:
        assert ((ro.double() - ref[0]).abs() <= ref[2] + R.rounding(ref[0], rt)).all()
    if has_out:
        assert ((out.double() - ref[1]).abs() <= ref[3] + R.rounding(ref[1], dt)).all()
    for v, b, old in ((ro, ro_buf, before[0]), (out, out_buf, before[1])):
        if b is not None:
            same_outside(v, b, old)
    h.destroy()


@pytest.mark.parametrize("d", [1, 2, 7, 8, 63, 64, 511, 512, 513, 1000, 1024, 1032, 2048, 4100, 7168, 8200, 16384])
@pytest.mark.parametrize("dtype,res", [("bf16", "bf16"), ("fp16", "fp32")])
def test_norm_widths(d, dtype, res):
    run_norm(5, d, dtype, res, post=True, gate="element", offset=1.0, seed=d)
    run_norm(1, d, dtype, res, seed=d + 1)


@pytest.mark.parametrize("t", [1, 2, 3, 31, 33, 600])
@pytest.mark.parametrize("dtype,res", [("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "one"])
def test_norm_rows_and_gates(t, dtype, res, gate):
    run_norm(t, 320, dtype, res, post=t % 2 == 0, gate=gate, seed=t)
    run_norm(t, 77, dtype, res, post=t % 2 == 1, gate=gate, seed=t)


@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (1, 0), (0, 1), (5, 3), (16, 4)])
@pytest.mark.parametrize("inplace", [False, True])
def test_norm_strides_alignment_and_in_place(pad, shift, inplace):
    for res in ("bf16", "fp32"):
        run_norm(37, 256, "bf16", res, post=True, gate="element", pad=pad, shift=shift, inplace=inplace, seed=pad)
        run_norm(9, 1536, "fp16", "fp16" if res == "bf16" else res, pad=pad, shift=shift, inplace=inplace, seed=pad)


@pytest.mark.parametrize("d", [200, 2048])
def test_norm_with_parts_left_out(d):
    for post in (False, True):
        run_norm(6, d, "bf16", "bf16", post=post, has_res=False)
        run_norm(6, d, "bf16", "fp32", post=post, has_out=False, gate="channel")
        run_norm(6, d, "fp16", "fp16", post=post, has_res_out=False, wp=False, wn=False, offset=1.0)
    run_norm(6, d, "bf16", "bf16", has_y=False)
    run_norm(6, d, "fp16", "fp32", has_y=False, has_res_out=False)


def test_norm_zero_rows_infinities_and_nan():
    """A row of zeros is 0 with an eps; an infinity or a NaN stays in its row."""
    h = D.FtDense()
    res = torch.ones(4, 512, device=DEV).bfloat16()
    y = torch.zeros_like(res)
    res[1], res[2, 5], y[3, 9] = 0, float("inf"), NAN
    out, ro = torch.empty_like(res), torch.empty_like(res)
    h.add_norm(y, res, ro, out, eps=1e-6)
    assert torch.isfinite(out[0]).all() and (out[1] == 0).all() and (out[0] - 1).abs().max() < 2 ** -7
    assert torch.isnan(out[2, 5]) and (out[2, :5] == 0).all() and torch.isnan(out[3]).all()
    assert torch.isinf(ro[2, 5]) and torch.isnan(ro[3, 9]) and torch.isfinite(ro[3, :9]).all()
    h.destroy()


# -------------------------------------------------------------------------------------------------------------- w4
def make_w4(n, k, group, dtype, zeros, seed, scale=None):
    g = gen(seed)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = ((0.5 + torch.rand(n, k // group, generator=g, device=DEV)) * (0.3 * k ** -0.5)).to(R.DT[dtype])
    z = torch.randint(0, 16, (n, k // group), generator=g, device=DEV, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def run_w4(t, n, k, group, dtype, *, zeros=False, bias=False, out32=False, x_pad=0, y_pad=0, y_shift=0, seed=0):
    g, dt = gen(seed), R.DT[dtype]
    h = D.FtDense()
    codes, scales, z = make_w4(n, k, group, dtype, zeros, seed)
    size = D.w4_bytes(n, k, group, zeros)
    image = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    w = h.w4_pack(codes, scales, z, image=image)
    assert (image[size:] == 0xA5).all()
    x = wide(t, k, x_pad, dt, g)[0]
    b = torch.randn(n, generator=g, device=DEV).to(dt) if bias else None
    out, buf = wide(t, n, y_pad, torch.float32 if out32 else dt, g, y_shift)
    before = buf.clone()
    h.w4(x, w, out, bias=b)
    assert h.sync_status() == 0
    ref, err = R.w4(x, R.w4_weights(codes, scales, z), b, out.dtype)
    assert ((out.double() - ref).abs() <= err + R.rounding(ref, out.dtype)).all()
    same_outside(out, buf, before)
    h.destroy()


@pytest.mark.parametrize("n", [1, 15, 16, 17, 127, 128, 129, 1000, 2051])
@pytest.mark.parametrize("t", [1, 3, 8, 9, 16, 17, 40])
def test_w4_rows_and_tokens(n, t):
    run_w4(t, n, 256, 128, "bf16", zeros=n % 2 == 0, bias=t % 2 == 0, out32=n % 3 == 0, seed=n + t)
    run_w4(t, n, 160, 32, "fp16", zeros=n % 2 == 1, bias=t % 2 == 1, out32=n % 3 == 1, seed=n + t)


@pytest.mark.parametrize("k,group", [(32, 32), (64, 32), (64, 64), (96, 32), (128, 128), (192, 64), (384, 128), (1056, 32), (2048, 128), (4096, 64), (7168, 128),
                                     (8192, 32), (16384, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_w4_depths_and_groups(k, group, dtype):
    for t, n in ((1, 272), (6, 40), (13, 300), (70, 150)):
        run_w4(t, n, k, group, dtype, zeros=t % 2 == 1, out32=t == 13, seed=k + t)
    run_w4(70, 150, k, group, dtype, zeros=True, out32=True, seed=k)


@pytest.mark.parametrize("t", [2, 16, 24, 40, 200])
def test_w4_deepest(t):
    run_w4(t, 70, 65536, 128, "bf16", zeros=True, out32=t in (24, 200), seed=t)
    run_w4(t, 1100, 65536, 32, "fp16", bias=True, seed=t)


@pytest.mark.parametrize("t", [1, 5, 12, 32, 33, 130, 300, 520])
@pytest.mark.parametrize("n,k,group,dtype,zeros", [(5120, 2048, 128, "bf16", False), (2048, 4096, 32, "fp16", True), (9001, 1024, 64, "bf16", True)])
def test_w4_wide(t, n, k, group, dtype, zeros):
    run_w4(t, n, k, group, dtype, zeros=zeros, seed=t)
    run_w4(t, n, k, group, dtype, zeros=not zeros, out32=True, bias=True, seed=t)


@pytest.mark.parametrize("x_pad,y_pad,y_shift", [(8, 0, 0), (64, 3, 1), (0, 1, 0), (24, 0, 1)])
def test_w4_strides(x_pad, y_pad, y_shift):
    """Elements behind a row of x (NaN here) are not read, those behind a row of y not written."""
    for t in (2, 11, 50, 200):
        run_w4(t, 333, 224, 32, "bf16", x_pad=x_pad, y_pad=y_pad, y_shift=y_shift, seed=t)
        run_w4(t, 333, 256, 64, "fp16", x_pad=x_pad, y_pad=y_pad, y_shift=y_shift, out32=True, seed=t)


@pytest.mark.parametrize("t", [3, 14, 60])
def test_w4_outliers_infinities_and_nan_stay_in_their_token(t):
    """Products are exact whatever the magnitudes; a NaN or an infinity reaches its own token's results only."""
    h = D.FtDense()
    codes, scales, _ = make_w4(300, 512, 128, "bf16", False, 5)
    w = h.w4_pack(codes, scales)
    x = torch.randn(t, 512, generator=gen(6), device=DEV)
    x[0] *= 1e30
    x[1, 7] = 1e6
    x = x.bfloat16()
    out = torch.empty(t, 300, device=DEV)
    h.w4(x, w, out)
    ref, err = R.w4(x, R.w4_weights(codes, scales, None), None, out.dtype)
    assert ((out.double() - ref).abs() <= err + R.rounding(ref, torch.float32)).all()
    x2 = x.clone()
    x2[0, 500], x2[2, 3] = float("inf"), NAN
    out2 = torch.empty_like(out)
    h.w4(x2, w, out2)
    keep = [i for i in range(t) if i not in (0, 2)]
    assert torch.equal(out[keep], out2[keep]) and torch.isnan(out2[2]).all() and not torch.isfinite(out2[0]).any()
    h.destroy()


def test_w4_zero_points_above_15_count_as_15():
    h = D.FtDense()
    codes, scales, z = make_w4(40, 128, 64, "fp16", True, 3)
    x = torch.randn(4, 128, generator=gen(1), device=DEV).half()
    a, b = torch.empty(4, 40, device=DEV), torch.empty(4, 40, device=DEV)
    z[::3] = 15
    h.w4(x, h.w4_pack(codes, scales, z), a)
    z[::3] = 200
    h.w4(x, h.w4_pack(codes, scales, z), b)
    assert torch.equal(a, b)
    h.destroy()


# ------------------------------------------------------------------------------------------------------------ logp
def run_logp(logits, k, scale=1.0, n=3, seed=0):
    h = D.FtDense()
    t, v = logits.shape
    tokens = torch.randint(0, v, (t, n), generator=gen(seed), device=DEV, dtype=torch.int32)
    f = lambda *s: torch.full(s, -77.0, device=DEV)
    lp, ent, top = f(t, n), f(t), f(t, k)
    ids = torch.full((t, k), -77, device=DEV, dtype=torch.int32)
    h.logprobs(logits, tokens=tokens, logprob=lp, entropy=ent, top_ids=ids if k else None, top_logprobs=top if k else None, scale=scale)
    assert h.sync_status() == 0
    logp, e, want, e_lp, e_ent = R.logprobs(logits, scale, k)

    def near(got, ref, tol):
        ok = ((got.double() - ref).abs() <= tol + R.rounding(ref, torch.float32)) | (got.double() == ref) | (torch.isnan(got) & torch.isnan(ref))
        assert ok.all()

    at = tokens.long()
    near(lp, logp.gather(1, at), e_lp.gather(1, at))
    near(ent, e, e_ent)
    if k:
        assert torch.equal(ids.long(), want)
        at = want.clamp(min=0)
        ref = logp.gather(1, at)
        ref = torch.where((want < 0) & ~torch.isnan(ref), -float("inf"), ref)
        near(top, ref, e_lp.gather(1, at))
    h.destroy()


@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 31, 33, 1000, 4096, 4099, 32003, 150000])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_logp_vocabularies(v, dtype):
    for t, k in ((1, 20), (3, 1), (40, 32)):
        run_logp((4 * torch.randn(t, v, generator=gen(v + t), device=DEV)).to(R.DT[dtype]), k, scale=0.7, seed=v)


@pytest.mark.parametrize("t", [1, 2, 18, 37, 74, 75, 148, 149, 297, 700])
def test_logp_rows(t):
    run_logp((3 * torch.randn(t, 9001, generator=gen(t), device=DEV)).bfloat16(), 7, seed=t)
    run_logp((3 * torch.randn(t, 40000, generator=gen(t), device=DEV)).half(), 0, seed=t)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 2), (5, 7)])
def test_logp_strides_and_alignment(dtype, pad, shift):
    for v in (5, 1003, 20000):
        run_logp(wide(6, v, pad, R.DT[dtype], gen(v), shift, scale=3.0)[0], 11, seed=shift)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t", [5, 310])
def test_logp_rows_of_every_kind(dtype, t):
    """Equal logits, ascending and descending ones, masks of -infinity and of the type's lowest value, rows that a mask leaves empty or with a few
    places, +infinity, NaN, large magnitudes, one certain token, alternatives that all stand where one thread reads."""
    dt, v = R.DT[dtype], 20001
    base = torch.randn(t, v, generator=gen(1), device=DEV)
    rows = []
    rows.append(torch.zeros(v, device=DEV))
    rows.append(torch.arange(v, device=DEV) / 100)
    rows.append(-torch.arange(v, device=DEV) / 100)
    low = torch.finfo(dt).min
    for fill in (-float("inf"), low):
        m = base[0].clone()
        m[torch.rand(v, generator=gen(2), device=DEV) < 0.99] = fill
        rows.append(m)
        m = torch.full((v,), fill, device=DEV)
        rows.append(m.clone())
        m[[3, 4000, 20000]] = torch.tensor([1.0, 2.0, 1.0], device=DEV)
        rows.append(m)
    for bad in (float("inf"), NAN):
        m = base[1].clone()
        m[777] = bad
        rows.append(m)
        m = torch.full((v,), -float("inf"), device=DEV)
        m[v - 1] = bad
        rows.append(m)
    rows.append(base[2] * 1e30)
    rows.append(torch.where(torch.arange(v, device=DEV) == 9999, 300.0, base[3]))
    m = base[4].clone()
    m[(torch.arange(v, device=DEV) // 8) % 512 == 5] += 30
    rows.append(m)
    m = torch.zeros(v, device=DEV)
    m[::7] = 1.0
    rows.append(m)
    for i, r in enumerate(rows):
        x = base.clone()
        x[t - 1 - i % t] = r
        run_logp(x.to(dt), 32 if i % 2 else 5, seed=i)


def test_logp_tokens_that_are_none_or_cannot_be():
    h = D.FtDense()
    x = torch.randn(4, 100, generator=gen(1), device=DEV)
    tokens = torch.tensor([[0, -1], [99, -5], [100, 1], [7, 2 ** 31 - 1]], dtype=torch.int32, device=DEV)
    lp = torch.empty(4, 2, device=DEV)
    h.logprobs(x, tokens=tokens, logprob=lp)
    assert h.sync_status() == B.FT_ERR_INVALID_ARG and h.sync_status() == 0
    assert lp[0, 1] == 0 and lp[1, 1] == 0 and torch.isnan(lp[2, 0]) and torch.isnan(lp[3, 1])
    assert torch.isfinite(lp[[0, 1, 2, 3], [0, 0, 1, 0]]).all()
    many = torch.randint(0, 100, (2, 1500), generator=gen(2), device=DEV, dtype=torch.int32)
    out = torch.empty(2, 1500, device=DEV)
    h.logprobs(x[:2], tokens=many, logprob=out)
    assert (out - torch.log_softmax(x[:2].double(), -1).gather(1, many.long())).abs().max() < 1e-5
    h.destroy()


# -------------------------------------------------------------------------------------------------------- refusals
def test_refusals():
    h = D.FtDense()
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d, device=DEV)
    y = z(4, 64)

    def refused(code, f):
        n = h.launch_count()
        with pytest.raises(D.FtDenseError) as e:
            f()
        assert e.value.code == code and h.launch_count() == n

    bad, no = B.FT_ERR_INVALID_ARG, B.FT_ERR_UNSUPPORTED
    refused(bad, lambda: h.add_norm(None, None, None, y))
    refused(bad, lambda: h.add_norm(y, None, None, None))
    refused(bad, lambda: h.add_norm(y, z(4, 65), None, y))
    refused(bad, lambda: h.add_norm(y, z(4, 64, d=torch.float16), None, y))
    refused(bad, lambda: h.add_norm(y.float(), y.float(), None, y.float()))
    refused(bad, lambda: h.add_norm(y, y, None, y, w_pre=z(63)))
    refused(bad, lambda: h.add_norm(y, y, None, y, gate=z(3, 64)))
    refused(bad, lambda: h.add_norm(y, y, None, y, eps=-1.0))
    refused(bad, lambda: h.add_norm(y, y, None, y, eps=NAN))
    refused(bad, lambda: h.add_norm(y.t().contiguous().t(), None, None, y))
    refused(bad, lambda: h.add_norm(y.cpu(), None, None, y))
    refused(no, lambda: h.add_norm(z(1, 16392), None, None, z(1, 16392)))
    codes, scales = z(40, 64, d=torch.uint8), z(40, 1)
    w = h.w4_pack(codes, scales)
    refused(no, lambda: h.w4_pack(codes, z(40, 8)))
    refused(no, lambda: h.w4_pack(codes, z(40, 3)))
    refused(bad, lambda: h.w4_pack(codes, z(40, 1, d=torch.float32)))
    refused(bad, lambda: h.w4_pack(codes, scales, zeros=z(40, 2, d=torch.uint8)))
    refused(bad, lambda: h.w4_pack(codes, scales, image=z(64, d=torch.uint8)))
    refused(bad, lambda: h.w4(z(2, 128, d=torch.float16), w, z(2, 40, d=torch.float16)))
    refused(bad, lambda: h.w4(z(2, 64), w, z(2, 40)))
    refused(bad, lambda: h.w4(z(2, 128), w, z(2, 41)))
    refused(bad, lambda: h.w4(z(2, 128), w, z(2, 40, d=torch.float16)))
    refused(bad, lambda: h.w4(z(2, 129)[:, :128], w, z(2, 40)))
    refused(bad, lambda: h.w4(z(257)[1:].view(2, 128), w, z(2, 40)))
    refused(bad, lambda: h.w4(z(2, 128), w, z(2, 40), bias=z(39)))
    x = z(2, 100)
    f = z(2, 1, d=torch.float32)
    i = z(2, 1, d=torch.int32)
    refused(bad, lambda: h.logprobs(x, tokens=i))
    refused(bad, lambda: h.logprobs(x, tokens=i.long(), logprob=f))
    refused(bad, lambda: h.logprobs(x, top_ids=i))
    refused(bad, lambda: h.logprobs(x, top_ids=z(2, 33, d=torch.int32), top_logprobs=z(2, 33, d=torch.float32)))
    refused(bad, lambda: h.logprobs(x, entropy=z(3, d=torch.float32)))
    for scale in (0.0, -1.0, NAN, float("inf")):
        refused(bad, lambda: h.logprobs(x, entropy=z(2, d=torch.float32), scale=scale))
    refused(bad, lambda: h.logprobs(x.to(torch.int32), entropy=z(2, d=torch.float32)))
    h.destroy()


def test_empty_calls():
    h = D.FtDense()
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d, device=DEV)
    h.add_norm(z(0, 64), z(0, 64), z(0, 64), z(0, 64))
    w = h.w4_pack(z(16, 32, d=torch.uint8), z(16, 1))
    n = h.launch_count()
    h.w4(z(0, 64), w, z(0, 16))
    h.logprobs(z(0, 64), entropy=z(0, d=torch.float32))
    assert h.launch_count() == n and h.sync_status() == 0
    h.destroy()
