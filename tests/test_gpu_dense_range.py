"""GPU tests of the operators of ``dense`` at the ends of what their arguments may hold: products of logit and scale far beyond the logits' usual ones."""
import pytest
import torch

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
