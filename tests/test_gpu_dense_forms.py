"""The forms of the kernels of ``dense`` that a size selects, each against the 64-bit form at sizes that select it; 4-bit products at tolerances that do not
grow with k; rows of inputs and results more than 2^32 bytes from their start."""
import pytest
import torch

from paper_2608_16157_b200 import dense as D
from tests import dense_reference as R
from tests.test_gpu_dense import DEV, gen, make_w4, run_logp, run_norm, run_w4

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------ norm
# more than 1.2 million elements: 16 of them a thread
@pytest.mark.parametrize("t,d", [(700, 2048), (5000, 320), (1300, 1000), (300, 7168), (170, 8192), (900, 1537), (20000, 77), (1200, 1031)])
@pytest.mark.parametrize("dtype,res", [("bf16", "bf16"), ("fp16", "fp32")])
@pytest.mark.parametrize("gate", ["none", "element", "channel", "token"])
def test_norm_of_many_elements(t, d, dtype, res, gate):
    run_norm(t, d, dtype, res, gate=gate, seed=d)
    run_norm(t, d, dtype, res, gate=gate, post=True, offset=1.0, inplace=True, seed=d + 1)


@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (16, 4)])
@pytest.mark.parametrize("res", ["fp16", "fp32"])
def test_norm_of_many_elements_strides_and_alignment(pad, shift, res):
    for post in (False, True):
        run_norm(800, 2048, "fp16", res, post=post, gate="element", pad=pad, shift=shift, seed=pad)
        run_norm(800, 2048, "fp16", res, post=post, pad=pad, shift=shift, inplace=True, seed=pad)
        run_norm(4000, 333, "fp16", res, post=post, gate="channel", pad=pad, shift=shift, seed=pad)


# ------------------------------------------------------------------------------------------------------------ logp
def odd_rows(x):
    """Some rows of equal logits, of a few places, of nothing, of NaN, of many equal largest ones."""
    t, v = x.shape
    x[1 % t] = 0.5
    x[3 % t, v // 3:] = -float("inf")
    x[5 % t] = -float("inf")
    x[7 % t, v - 1] = float("nan")
    x[9 % t, ::3] = 9.0
    return x


@pytest.mark.parametrize("t", [149, 200, 2049])
@pytest.mark.parametrize("dtype,vocabularies", [("bf16", (1, 7, 33, 1000, 4099, 8192)), ("fp16", (5, 1003, 8190)), ("fp32", (2, 130, 1000, 4096))])
def test_logp_many_rows_of_short_vocabularies(t, dtype, vocabularies):
    """More rows than SMs, at most 1024 pieces of 16 bytes: blocks of 128 threads."""
    for v in vocabularies:
        for k in (1, 8, 32):
            run_logp(odd_rows(3 * torch.randn(t, v, generator=gen(v + k), device=DEV)).to(R.DT[dtype]), k, scale=0.9, seed=k)


@pytest.mark.parametrize("t", [149, 200, 296, 297])
@pytest.mark.parametrize("dtype,v", [("bf16", 16384), ("bf16", 50001), ("fp16", 32003), ("fp32", 8200), ("fp32", 40000)])
def test_logp_pairs_of_blocks_with_alternatives(t, dtype, v):
    """Between one and two rows to a place, at least 2048 pieces: pairs of blocks of 256 threads (297 rows: one each)."""
    for k in (1, 5, 32):
        x = odd_rows(3 * torch.randn(t, v, generator=gen(v + k), device=DEV))
        x[11, v // 2 - 40:v // 2 + 40] += 20                        # the alternatives on both sides of the middle
        x[13, :] = torch.arange(v, device=DEV).float() * (40.0 / v)
        run_logp(x.to(R.DT[dtype]), k, seed=k)


# -------------------------------------------------------------------------------------------------------------- w4
# few tokens, more quads of 64 rows than groups of warps: one, four, eight warps to a quad, blocks of a cluster
@pytest.mark.parametrize("t,n,k,group,out32", [
    (3, 44800, 4096, 128, False), (8, 20000, 7168, 64, True), (12, 44800, 4096, 32, False), (16, 150001, 1024, 64, True), (13, 300000, 256, 128, False),
    (20, 20000, 4096, 64, True), (32, 44800, 2048, 128, True), (29, 44800, 4096, 32, True), (17, 150001, 256, 32, True), (25, 300000, 256, 64, True),
    (5, 13000, 65536, 128, False), (11, 13000, 65536, 64, True), (24, 7000, 65536, 128, True)])
@pytest.mark.parametrize("zeros", [False, True])
def test_w4_groups_of_warps_with_several_quads(t, n, k, group, out32, zeros):
    run_w4(t, n, k, group, "bf16" if zeros else "fp16", zeros=zeros, bias=zeros, out32=out32, seed=t)


@pytest.mark.parametrize("t,n,k,group", [(1, 300, 4096, 128), (7, 1100, 7168, 64), (14, 200, 65536, 128), (30, 200, 8192, 32), (17, 300, 7168, 128), (64, 150, 16384, 32),
                                         (200, 1100, 4096, 64), (300, 70, 65536, 128), (520, 5120, 2048, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("out32", [False, True])
def test_w4_every_group_of_k_counts(t, n, k, group, dtype, out32):
    """Tokens that see one group of k each, all groups in turn: the tolerance is of that group's products, a group that is missing, taken twice or scaled by
    another's scale is all of the result."""
    h, dt = D.FtDense(), R.DT[dtype]
    codes, scales, z = make_w4(n, k, group, dtype, True, k)
    scales *= torch.where(torch.arange(k // group, device=DEV) % 2 == 0, 1.0, -3.0).to(dt)      # (neighbours' scales differ)
    w, w64 = h.w4_pack(codes, scales, z), R.w4_weights(codes, scales, z)
    groups = k // group
    for start in range(0, groups, t):
        x = torch.zeros(t, groups, group, dtype=dt, device=DEV)
        at = (torch.arange(t, device=DEV) + start) % groups
        x[torch.arange(t, device=DEV), at] = (1 + torch.rand(t, group, generator=gen(start), device=DEV)).to(dt)
        x = x.view(t, k)
        y = torch.full((t, n), float("nan"), dtype=torch.float32 if out32 else dt, device=DEV)
        h.w4(x, w, y)
        ref, err = R.w4(x, w64, None, y.dtype)
        assert ((y.double() - ref).abs() <= err + R.rounding(ref, y.dtype)).all()
    assert h.sync_status() == 0
    h.destroy()


@pytest.mark.parametrize("t,n,k,group", [(17, 300, 7168, 128), (64, 1100, 2048, 32), (200, 1100, 4096, 64), (40, 320, 65536, 128), (512, 5120, 2048, 128), (300, 3000, 1024, 32)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("zeros", [False, True])
def test_w4_error_of_rounded_weights(t, n, k, group, dtype, zeros):
    """More than 16 tokens, 16-bit results: the error as a whole, of every token and of every tile of 16 rows.  A rounding is off by an amount spread evenly
    up to half a step, which is UNIT of the value at most: UNIT / sqrt(3) root mean square.  Those of k weights with signs of their own are to the
    result as one of them is to its weight; the result's own comes on top: UNIT sqrt(2 / 3).  The float sums: k / 16 additions, each off by 2^-22 of a
    partial sum at most.  (Over 270 and more values the measured root mean square is off by a few per cent; values within a binade keep it a third below.)"""
    h, dt = D.FtDense(), R.DT[dtype]
    codes, scales, z = make_w4(n, k, group, dtype, zeros, k)
    x = torch.randn(t, k, generator=gen(t), device=DEV).to(dt)
    y = torch.empty(t, n, dtype=dt, device=DEV)
    h.w4(x, h.w4_pack(codes, scales, z), y)
    ref = x.double() @ R.w4_weights(codes, scales, z).t()
    err = y.double() - ref
    tol = R.UNIT[dt] * (2 / 3) ** 0.5 + k / 16 * 2.0 ** -22
    assert (err.norm(dim=1) <= tol * ref.norm(dim=1)).all()
    tiles = [(err[:, i:i + 16].norm(), ref[:, i:i + 16].norm()) for i in range(0, n - 15, 16)]
    assert all(float(e) <= tol * float(r) for e, r in tiles)
    h.destroy()


@pytest.mark.parametrize("t,out32", [(5, False), (12, True), (24, True), (40, False), (40, True)])
def test_w4_rows_beyond_32_bit_offsets(t, out32):
    """Rows of x and of y that stand more than 2^32 bytes apart in all."""
    h, k, n = D.FtDense(), 512, 300
    codes, scales, z = make_w4(n, k, 128, "bf16", True, 1)
    room = (6 << 30) // (2 * t) // 64 * 64
    x = torch.zeros(t * room, dtype=torch.bfloat16, device=DEV).view(t, room)[:, -k:]
    y = torch.zeros(t * room, dtype=torch.float32 if out32 else torch.bfloat16, device=DEV).view(t, room)[:, -n:]
    assert (t - 1) * x.stride(0) * 2 > 1 << 32 and (t - 1) * y.stride(0) * y.element_size() > 1 << 32
    x.copy_(torch.randn(t, k, generator=gen(2), device=DEV))
    h.w4(x, h.w4_pack(codes, scales, z), y)
    ref, err = R.w4(x.contiguous(), R.w4_weights(codes, scales, z), None, y.dtype)
    assert ((y.double() - ref).abs() <= err + R.rounding(ref, y.dtype)).all()
    assert h.sync_status() == 0
    h.destroy()


def test_norm_rows_beyond_32_bit_offsets():
    h, g = D.FtDense(), gen(1)
    t, d, room = 600, 2048, 4_000_000                              # 4.8 GB a tensor, 9.6 the stream
    rows = lambda dt: torch.zeros(t * room, dtype=dt, device=DEV).view(t, room)[:, 1_000_000:1_000_000 + d]
    y, gate, out, res = rows(torch.bfloat16), rows(torch.bfloat16), rows(torch.bfloat16), rows(torch.float32)
    for x in (y, gate, res):
        x.copy_(torch.randn(t, d, generator=g, device=DEV))
    ref = R.add_norm(y, res, gate, None, None, post=True, w_offset=0.0, eps=1e-6, res_scale=1.0, y_scale=1.0)
    h.add_norm(y, res, res, out, gate=gate, post=True)
    assert ((res.double() - ref[0]).abs() <= ref[2] + R.rounding(ref[0], torch.float32)).all()
    assert ((out.double() - ref[1]).abs() <= ref[3] + R.rounding(ref[1], torch.bfloat16)).all()
    assert h.sync_status() == 0
    h.destroy()
