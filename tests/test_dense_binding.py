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
