"""Streams of the operators of ``dense``: an image that is made on one stream and written on another."""
import pytest
import torch

from paper_2608_16157_b200 import dense as D
from tests.test_gpu_dense import DEV, gen, make_w4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("raw", [False, True])
def test_an_image_packed_on_another_stream(raw):
    """The image's memory was another tensor's, to which queued work of the current stream still writes; and it is given back, and taken again,
    while the pack has not run yet."""
    h, st = D.FtDense(), torch.cuda.Stream()
    parts = make_w4(1000, 2048, 128, "bf16", True, 1)
    want = h.w4_pack(*parts).image
    size = want.numel()
    torch.cuda.synchronize()

    old = torch.empty(size, dtype=torch.uint8, device=DEV)
    at = old.data_ptr()
    torch.cuda._sleep(50_000_000)
    old.fill_(0xFF)
    del old
    w = h.w4_pack(*parts, stream=st.cuda_stream if raw else st)
    assert w.image.data_ptr() == at                     # (else this shows nothing)
    torch.cuda.synchronize()
    assert torch.equal(w.image, want)

    with torch.cuda.stream(st):
        torch.cuda._sleep(50_000_000)
    w = h.w4_pack(*parts, stream=st.cuda_stream if raw else st)
    del w
    new = torch.full((size,), 0x3C, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    assert (new == 0x3C).all()
    assert h.sync_status() == 0
    h.destroy()


def test_an_image_packed_on_the_current_stream_given_by_name():
    h = D.FtDense()
    parts = make_w4(100, 256, 64, "fp16", False, 1)
    want = h.w4_pack(*parts).image
    assert torch.equal(h.w4_pack(*parts, stream=torch.cuda.current_stream()).image, want)
    own = torch.empty_like(want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    assert h.w4_pack(*parts, image=own, stream=st).image is own
    st.synchronize()
    assert torch.equal(own, want)
    h.destroy()
