"""The part of the library behind include/ftdense.h: symbols, sizes of images, refusals that need no GPU."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_16157_b200 import binding as B
from paper_2608_16157_b200 import dense as D

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ftdense.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(ft_dense_[a-z_0-9]+)\s*\(", text)))
    lib = D.load()
    assert sorted(D.SYMBOLS) == declared
    for name in declared:
        assert hasattr(lib, name), name


@pytest.mark.parametrize("n,k,group,zeros,size", [
    (16, 64, 64, False, 1024 + 256), (1, 32, 32, False, 1024 + 512), (17, 128, 128, True, 2048 + 192), (130, 160, 32, True, 2 * (2 * (4096 + 768) + 1024 + 768)),
    (5120, 2048, 128, False, 5120 * 1024 + 5120 * 16 * 2),
])
def test_bytes_of_an_image(n, k, group, zeros, size):
    assert D.w4_bytes(n, k, group, zeros) == size


@pytest.mark.parametrize("n,k,group", [(0, 64, 64), (16, 64, 128), (16, 96, 64), (16, 64, 16), (16, 64, 0), (16, 0, 32), (16, 65536 + 128, 128), (1 << 25, 64, 64),
                                       (-1, 64, 64), (16, -64, 64), (1 << 40, 64, 64)])
def test_shapes_without_an_image(n, k, group):
    assert D.w4_bytes(n, k, group) == 0


def test_null_handles_are_refused():
    lib = D.load()
    z = (None,) * 20
    assert lib.ft_dense_create(0, None) == B.FT_ERR_INVALID_ARG
    h = ctypes.c_void_p()
    assert lib.ft_dense_create(-1, ctypes.byref(h)) == B.FT_ERR_INVALID_ARG and not h.value
    assert lib.ft_dense_destroy(None) == B.FT_OK
    assert lib.ft_dense_sync_status(None) == B.FT_ERR_INVALID_ARG
    assert lib.ft_dense_add_norm(None, 1, 8, 0, 0, 0, None, 8, None, 8, None, 0, 0, None, None, 0.0, 0.0, 1.0, 1.0, None, 8, None, 8, None) == B.FT_ERR_INVALID_ARG
    assert lib.ft_dense_w4_pack(None, 16, 64, 64, 0, None, 32, *z[:4]) == B.FT_ERR_INVALID_ARG
    assert lib.ft_dense_w4_forward(None, 1, 16, 64, 64, 0, 0, None, 64, None, None, None, 16, 0, None) == B.FT_ERR_INVALID_ARG
    assert lib.ft_dense_logprobs(None, 1, 8, 0, None, 8, 1.0, None, 0, 0, None, None, 0, None, None, None) == B.FT_ERR_INVALID_ARG
    n = ctypes.c_uint64()
    assert lib.ft_dense_launch_count(None, ctypes.byref(n)) == B.FT_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype,bits,base", [(torch.bfloat16, lambda i: 3 + 4 * i if i < 3 else 15, 3), (torch.float16, lambda i: (6, 10, 2, 14)[i], 6)])
def test_where_the_nibbles_of_a_word_stand(dtype, bits, base):
    """The layout's arithmetic: the eight nibbles of a word are disjoint, and a shift or rotation brings each pair to the mantissa's top."""
    magic = 0x4180 if dtype is torch.bfloat16 else 0x4C00
    rot = lambda v, n: ((v << n) | (v >> (32 - n))) & 0xFFFFFFFF if n else v
    used = 0
    for i in range(4):
        for half in range(2):
            m = rot(15, (bits(i) + 16 * half) % 32)
            assert used & m == 0
            used |= m
    assert used == 0xFFFFFFFF
    word = 0
    for i in range(4):
        for half in range(2):
            word |= rot(2 * i + 7 * half, (bits(i) + 16 * half) % 32)
    for i in range(4):
        p = rot(word, (32 - bits(i) + base) % 32) & (15 << base | 15 << (base + 16)) | magic | magic << 16
        for half in range(2):
            v = torch.tensor((p >> 16 * half) & 0xFFFF, dtype=torch.int32).to(torch.int16).view(dtype)
            assert float(v) == 16 + 2 * i + 7 * half
