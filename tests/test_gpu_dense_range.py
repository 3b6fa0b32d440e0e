"""GPU tests of the operators of ``dense`` at the ends of what their arguments may hold: products of logit and scale far beyond the logits' usual ones,
scales and logits next to the smallest and the largest floats."""
import pytest
import torch

from paper_2608_16157_b200 import binding as B
from paper_2608_16157_b200 import dense as D
from tests import dense_reference as R
from tests.test_gpu_dense import DEV, gen, run_logp

pytestmark = pytest.mark.gpu


# (type, what masked places hold, scale): the largest product of logit and scale is 2^30 and more, where rounding it loses whole units
FILLS = [("bf16", -1e9, 1.0), ("bf16", -1e10, 0.8), ("bf16", -1e12, 1.0), ("bf16", -1e20, 1.0), ("bf16", -40.0, 1e7), ("fp32", -1e9, 0.7), ("fp32", -1e10, 1.0),
         ("fp32", -1e12, 1.0), ("fp32", -1e20, 3.0), ("fp32", -1e4, 3e7), ("fp16", -1000.0, 1e6), ("fp16", -60000.0, 1e5), ("fp16", -65504.0, 1e7),
         ("fp16", -65504.0, 1e-3), ("fp16", -float("inf"), 1.0)]


@pytest.mark.parametrize("dtype,fill,scale", FILLS)
@pytest.mark.parametrize("t,v", [(1, 150000), (5, 20001), (200, 40000)])
def test_logp_rows_filled_with_a_finite_mask(dtype, fill, scale, t, v):
    """Rows of nothing but the mask's value, rows with a few places left, one eighth of the vocabulary left (what one block of a row sees is all masked),
    and rows whose largest logit is as far above zero."""
    base = torch.randn(t, v, generator=gen(1), device=DEV)
    rows = [torch.full((v,), fill, device=DEV) for _ in range(6)]
    rows[1][[1, v // 3, v - 1]] = torch.tensor([1.0, 2.0, 1.0], device=DEV)
    rows[2][v // 2:v // 2 + v // 8] = base[0, :v // 8]
    rows[3][:v // 8] = base[0, :v // 8]
    if fill != -float("inf"):
        rows[4] = -rows[4]
        rows[5] = base[0].clone()
        rows[5][v - 7] = -fill
    for i, r in enumerate(rows):
        x = base.clone()
        x[t - 1 - i % t] = r
        run_logp(x.to(R.DT[dtype]), (7, 0, 32)[i % 3], scale=scale, seed=i)


@pytest.mark.parametrize("dtype,big", [("bf16", 1e10), ("bf16", 1e20), ("fp32", 1e10), ("fp32", 1e20), ("fp32", 3e7)])
@pytest.mark.parametrize("t,v", [(1, 60000), (3, 9001), (300, 5000)])
def test_logp_maxima_far_from_zero(dtype, big, t, v):
    """Logits that differ by the type's steps at a magnitude far above one, above and below zero."""
    dt = R.DT[dtype]
    for sign in (1.0, -1.0):
        step = big * torch.finfo(dt).eps
        x = sign * big + step * torch.randint(-4, 5, (t, v), generator=gen(3), device=DEV)
        for scale in (1.0, 1.0 / step, 3.0 / big):
            run_logp(x.to(dt), 12, scale=scale, seed=v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("exponent", [-149, -131, -128, -126, -120])
@pytest.mark.parametrize("t,v", [(1, 60000), (4, 801), (300, 5000)])
def test_logp_differences_beyond_the_largest_float(dtype, exponent, t, v):
    """Logits over the whole range of the type, the largest and the lowest value among them, times a scale that leaves ordinary differences."""
    low, high = torch.finfo(R.DT[dtype]).min, torch.finfo(R.DT[dtype]).max
    x = (2 * torch.rand(t, v, generator=gen(4), device=DEV) - 1) * 3e38
    x[:, 5], x[:, v - 9] = low, high
    x[0, v // 2:] = low
    run_logp(x.to(R.DT[dtype]), 9, scale=2.0 ** exponent, seed=t)


@pytest.mark.parametrize("dtype,size,exponent", [("fp32", 2.0 ** -125, 126), ("fp32", 2.0 ** -140, 126), ("bf16", 2.0 ** -124, 126), ("fp32", 1.0, 100), ("fp16", 1.0, 100),
                                                 ("bf16", 2.0 ** -100, 105)])
@pytest.mark.parametrize("t,v", [(1, 60000), (4, 801), (300, 5000)])
def test_logp_the_largest_scales(dtype, size, exponent, t, v):
    run_logp((size * torch.randn(t, v, generator=gen(5), device=DEV)).to(R.DT[dtype]), 9, scale=2.0 ** exponent, seed=t)


def test_logp_scales_beyond_the_largest_are_refused():
    h = D.FtDense()
    x, e = torch.zeros(2, 100, device=DEV), torch.full((2,), -77.0, device=DEV)
    for scale in (1.01 * 2.0 ** 126, 2.0 ** 127, 3e38):
        with pytest.raises(D.FtDenseError) as err:
            h.logprobs(x, entropy=e, scale=scale)
        assert err.value.code == B.FT_ERR_INVALID_ARG
    assert h.launch_count() == 0 and (e == -77).all()
    h.logprobs(x, entropy=e, scale=2.0 ** 126)
    assert (e - 4.605170186).abs().max() < 1e-5
    h.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,v", [(300, 87103), (20, 60001)])
def test_logp_entropy_of_rows_of_one_far_value(dtype, t, v):
    """Every row holds one value of its own between -1e7 and -1e9: the logarithm of the vocabulary to float's accuracy, whatever the products lost."""
    x = -(10.0 ** torch.linspace(7, 9, t, device=DEV))[:, None].expand(t, v)
    run_logp(x.to(R.DT[dtype]).contiguous(), 3, seed=t)
