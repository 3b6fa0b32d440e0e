"""``add_norm`` at the ends of what its arguments may hold."""
import pytest
import torch

from paper_2608_16157_b200 import dense as D
from tests import dense_reference as R
from tests.test_gpu_dense import DEV, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("res", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("t,d", [(1, 5), (7, 512), (300, 2048)])
def test_a_stream_alone(res, t, d):
    """Neither a block's output nor a norm: the stream is scaled."""
    h = D.FtDense()
    r = torch.randn(t, d, generator=gen(1), device=DEV).to(R.DT[res])
    want = 0.7 * r.double()
    out = torch.empty_like(r)
    h.add_norm(None, r, out, None, res_scale=0.7)
    h.add_norm(None, r, r, None, res_scale=0.7)
    assert torch.equal(out, r)
    # (0.7 as a float is off by 2^-25, the product by 2^-24)
    assert ((r.double() - want).abs() <= 2.0 ** -23 * want.abs() + R.rounding(want, r.dtype)).all()
    assert h.sync_status() == 0 and h.launch_count() == 2
    h.destroy()


def test_as_many_rows_as_there_can_be():
    h = D.FtDense()
    t = 2 ** 31 - 1
    y = torch.empty(t, 1, dtype=torch.bfloat16, device=DEV)
    y[::2], y[1::2] = 3.0, -2.0
    out = torch.zeros_like(y)
    h.add_norm(y, None, None, out, eps=0.0, y_scale=2.0)
    assert h.sync_status() == 0
    assert (out[::2] == 1).all() and (out[1::2] == -1).all()
    h.destroy()


@pytest.mark.parametrize("size,eps", [(1e20, 1e-6), (1e30, 0.0), (3e36, 1e-6), (1e-18, 0.0), (1e-25, 0.0), (1e-25, 2.0 ** -149), (1e-25, 1e-38), (1e-36, 0.0), (1e-39, 0.0), (1e-20, 1e-24),
                                      (1e-30, 1e-30), (1e18, 1e30)])
@pytest.mark.parametrize("t,d", [(3, 1), (5, 77), (9, 320), (4, 2048), (2, 8200), (900, 1537), (700, 2048)])
@pytest.mark.parametrize("dtype,res", [("bf16", "bf16"), ("bf16", "fp32")])
def test_rows_whose_squares_leave_the_range_of_float(size, eps, t, d, dtype, res):
    """Rows of large and of small magnitude, an ordinary one and one of zeros (with an eps) among them: all are normed like the others."""
    h, g = D.FtDense(), gen(d)
    dt, rt = R.DT[dtype], R.DT[res]
    for post in (False, True, "apart"):
        y = (size * torch.randn(t, d, generator=g, device=DEV).clamp(-8, 8)).to(dt)
        r = (size * torch.randn(t, d, generator=g, device=DEV).clamp(-8, 8)).to(rt)
        if t > 2:
            y[1], r[1] = 1.5, -0.25
            if eps:
                y[2], r[2] = 0, 0
        w = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt)
        gate = torch.randn(t, d, generator=g, device=DEV).to(dt) if d % 2 else None
        if post:                                         # (beside what is normed: the stream over the size, infinite where that is below 1 / 3e38; another)
            r = (r.float() / size).to(rt) if post is True else torch.randn(t, d, generator=g, device=DEV).to(rt)
            post = True
        ref = R.add_norm(y, r, gate, w if post else None, w, post=post, w_offset=0.5, eps=eps, res_scale=0.9, y_scale=0.7)
        ro, out = torch.empty_like(r), torch.empty_like(y)
        h.add_norm(y, r, ro, out, post=post, w_post=w if post else None, w_pre=w, gate=gate, w_offset=0.5, eps=eps, res_scale=0.9, y_scale=0.7)
        # two products and a sum that fall on subnormal numbers are off by 2^-150 each: 2^-148 of r', and that over the root mean square in h
        cut = 2.0 ** -148
        near = (ro.double() - ref[0]).abs() <= ref[2] + cut + R.rounding(ref[0], rt)
        assert (near | (ro.double() == ref[0]) | torch.isnan(ro) & torch.isnan(ref[0])).all()
        inv = 1 / torch.sqrt((ref[0] ** 2).mean(-1, keepdim=True) + eps)
        tol = ref[3] + cut * inv * ((0.5 + w.double()).abs() + ref[1].abs())
        assert (((out.double() - ref[1]).abs() <= tol + R.rounding(ref[1], dt)) | torch.isnan(out) & torch.isnan(ref[1])).all()
    assert h.sync_status() == 0
    h.destroy()


def test_a_row_of_zeros_without_an_eps_is_not_a_number():
    h = D.FtDense()
    out = torch.zeros(2, 64, dtype=torch.bfloat16, device=DEV)
    h.add_norm(None, torch.zeros(2, 64, device=DEV), None, out, eps=0.0)
    assert torch.isnan(out).all()
    h.destroy()


@pytest.mark.parametrize("t,d", [(4, 320), (700, 2048)])
def test_an_infinite_eps_leaves_nothing(t, d):
    h = D.FtDense()
    y = (1e30 * torch.randn(t, d, generator=gen(1), device=DEV)).bfloat16()
    out, ro = torch.ones_like(y), torch.ones_like(y)
    h.add_norm(y, None, ro, out, eps=float("inf"))
    assert (out == 0).all() and torch.equal(ro, y)
    h.add_norm(y, None, ro, out, eps=float("inf"), post=True)
    assert (out == 0).all() and (ro == 0).all()
    h.destroy()
