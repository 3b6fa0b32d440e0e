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
