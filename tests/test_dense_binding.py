"""Host side of the binding of ``dense`` that needs no GPU: which device a handle is for, refusals."""
import pytest
import torch

from paper_2608_16157_b200 import binding as B
from paper_2608_16157_b200 import dense as D


@pytest.mark.parametrize("device,index", [(None, 3), ("cuda", 3), (torch.device("cuda"), 3), ("cuda:0", 0), ("cuda:5", 5), (torch.device("cuda", 2), 2), (0, 0), (4, 4)])
def test_the_device_of_a_handle(monkeypatch, device, index):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    asked = []

    class Lib:
        def ft_dense_create(self, i, out):
            asked.append(i)
            return B.FT_ERR_CUDA

        def ft_dense_last_cuda_error(self):
            return b"none here"

    monkeypatch.setattr(D, "load", Lib)
    with pytest.raises(D.FtDenseError):
        D.FtDense(device)
    assert asked == [index]


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), "meta"])
def test_a_device_that_is_none(device):
    with pytest.raises(D.FtDenseError) as e:
        D.FtDense(device)
    assert e.value.code == B.FT_ERR_INVALID_ARG


@pytest.fixture
def handle():
    """A handle of CPU tensors' "device": its checks run, its library must not be reached."""
    h = D.FtDense.__new__(D.FtDense)
    h._h, h._lib, h._index, h._device = None, None, -1, torch.device("cpu")
    return h


def test_calls_without_a_tensor_are_refused(handle):
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d)
    w = D.W4Weight(z(64, d=torch.uint8), 16, 32, 32, torch.bfloat16, False)
    for call in (lambda: handle.add_norm(None, None, None, None), lambda: handle.add_norm(None, None, None, None, w_pre=z(8)),
                 lambda: handle.add_norm(None, None, None, None, w_post=z(8), post=True), lambda: handle.add_norm(z(8), None, None, z(8)),
                 lambda: handle.add_norm(torch.zeros(()), None, None, None), lambda: handle.w4(torch.zeros((), dtype=torch.bfloat16), w, z(1, 16)),
                 lambda: handle.w4(z(32), w, z(16)), lambda: handle.w4(z(1, 1, 32), w, z(1, 16)), lambda: handle.logprobs(z(8)),
                 lambda: handle.logprobs(torch.zeros(()))):
        with pytest.raises(D.FtDenseError) as e:
            call()
        assert e.value.code == B.FT_ERR_INVALID_ARG
