"""4-bit products whose scales reach the ends of their type: weights that the type cannot hold, weights below its normal numbers."""
import pytest
import torch

from paper_2608_16157_b200 import dense as D
from tests import dense_reference as R
from tests.test_gpu_dense import DEV, gen, make_w4

pytestmark = pytest.mark.gpu


def run(t, n, k, group, dtype, zeros, change, size, bias=False, seed=0):
    """Products of x of the given size with a matrix whose scales `change` has altered, as 16-bit results, against the 64-bit form."""
    g, dt = gen(seed), R.DT[dtype]
    h = D.FtDense()
    codes, scales, z = make_w4(n, k, group, dtype, zeros, seed)
    change(scales)
    x = (size * torch.randn(t, k, generator=g, device=DEV)).to(dt)
    x[t // 2] = 0
    b = torch.randn(n, generator=g, device=DEV).to(dt) if bias else None
    y = torch.full((t, n), float("nan"), dtype=dt, device=DEV)
    h.w4(x, h.w4_pack(codes, scales, z), y, bias=b)
    assert h.sync_status() == 0
    ref, err = R.w4(x, R.w4_weights(codes, scales, z), b, dt)
    assert torch.isfinite(y).all()
    assert ((y.double() - ref).abs() <= err + R.rounding(ref, dt)).all()
    assert (y[t // 2] == (0 if b is None else b)).all()
    h.destroy()


@pytest.mark.parametrize("t", [3, 16, 17, 40, 130, 500])
@pytest.mark.parametrize("n,k,group,zeros", [(200, 512, 128, False), (333, 1056, 32, True), (1100, 192, 64, True), (70, 4096, 64, False), (9000, 256, 32, True)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_weights_that_the_type_cannot_hold(t, n, k, group, zeros, dtype):
    """Scales up to the type's largest value in some groups, both signs: weights are infinite in the type, results are not, whatever the number of tokens."""
    top = torch.finfo(R.DT[dtype]).max

    def some(scales):
        s = torch.rand(scales.shape, generator=gen(9), device=DEV)
        scales[s < 0.03] = top / 10
        scales[s < 0.02] = -top / 4
        scales[s < 0.01] = top
        scales[0], scales[-1, -1] = top, -top                 # a whole row; the last group

    run(t, n, k, group, dtype, zeros, some, 6e-6 if dtype == "fp16" else 1e-4, bias=t % 2 == 0, seed=t)


@pytest.mark.parametrize("t", [16, 40, 300])
@pytest.mark.parametrize("zeros", [False, True])
def test_weights_below_the_normal_numbers(t, zeros):
    """A product of a subnormal scale and a code difference is a multiple of the type's smallest step: nothing is lost."""
    def small(scales):
        scales.copy_((scales.float() * 2.0 ** -8).to(scales.dtype))
        scales[::3] = 2.0 ** -24

    run(t, 300, 512, 64, "fp16", zeros, small, 1.0, seed=t)


def test_a_nan_token_beside_weights_that_the_type_cannot_hold():
    """Only the token's own results are NaN."""
    h = D.FtDense()
    codes, scales, _ = make_w4(300, 512, 128, "fp16", False, 2)
    scales[5], scales[7, 2] = 60000.0, 30000.0
    w = h.w4_pack(codes, scales)
    x = (1e-5 * torch.randn(50, 512, generator=gen(3), device=DEV)).half()
    y = torch.empty(50, 300, dtype=torch.float16, device=DEV)
    h.w4(x, w, y)
    clean = y.clone()
    x[20, 9], x[33, 500] = float("nan"), float("inf")
    h.w4(x, w, y)
    keep = [i for i in range(50) if i not in (20, 33)]
    assert torch.isfinite(clean).all() and torch.equal(y[keep], clean[keep])
    assert torch.isnan(y[20]).all() and not torch.isfinite(y[33]).any()
    h.destroy()
