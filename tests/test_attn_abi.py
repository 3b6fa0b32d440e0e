"""The attention operators' part of the library: symbols, configuration checks, refusals that need no GPU."""
import ctypes
import os
import re

import pytest

from paper_2608_16157_b200 import attention as A
from paper_2608_16157_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GOOD = dict(n_q_heads=32, n_kv_heads=4, head_dim=128, page_tokens=16, n_pages=64, max_requests=8, max_tokens=64, max_pages=8)


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ftattn.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(ft_attn_[a-z_0-9]+)\s*\(", text)))
    lib = A.load()
    assert sorted(A.SYMBOLS) == declared
    for name in declared:
        assert hasattr(lib, name), name


def test_config_size_and_cache_bytes():
    assert ctypes.sizeof(A.Config) == 12 * 4
    assert A.cache_bytes(A.make_config(**GOOD)) == 64 * 2 * 4 * 16 * 128 * 2
    assert A.cache_bytes(A.make_config(**{**GOOD, "head_dim": 96})) == 0


@pytest.mark.parametrize("change,code", [
    (dict(n_kv_heads=3), B.FT_ERR_INVALID_ARG), (dict(n_kv_heads=0), B.FT_ERR_INVALID_ARG),
    (dict(n_q_heads=260, n_kv_heads=4), B.FT_ERR_INVALID_ARG), (dict(head_dim=96), B.FT_ERR_UNSUPPORTED),
    (dict(page_tokens=24), B.FT_ERR_UNSUPPORTED), (dict(n_pages=0), B.FT_ERR_INVALID_ARG), (dict(n_pages=1 << 27), B.FT_ERR_INVALID_ARG),
    (dict(max_requests=0), B.FT_ERR_INVALID_ARG), (dict(max_requests=1025), B.FT_ERR_INVALID_ARG),
    (dict(max_tokens=0), B.FT_ERR_INVALID_ARG), (dict(max_pages=1 << 28), B.FT_ERR_INVALID_ARG), (dict(window=-1), B.FT_ERR_INVALID_ARG),
    (dict(device=-1), B.FT_ERR_INVALID_ARG), (dict(max_pages=1 << 26, max_requests=1024), B.FT_ERR_UNSUPPORTED),
])
def test_create_refuses_without_a_gpu_call(change, code):
    cfg = A.make_config(**{**GOOD, **change})
    h = ctypes.c_void_p()
    assert A.load().ft_attn_create(ctypes.byref(cfg), ctypes.byref(h)) == code
    assert not h.value


def test_null_handles_and_a_wrong_struct_size_are_refused():
    lib = A.load()
    h = ctypes.c_void_p()
    cfg = A.make_config(**GOOD)
    cfg.struct_size = 3
    assert lib.ft_attn_create(ctypes.byref(cfg), ctypes.byref(h)) == B.FT_ERR_INVALID_ARG
    assert lib.ft_attn_create(None, ctypes.byref(h)) == B.FT_ERR_INVALID_ARG
    assert lib.ft_attn_create(ctypes.byref(cfg), None) == B.FT_ERR_INVALID_ARG
    assert lib.ft_attn_destroy(None) == B.FT_OK
    z = (None,) * 20
    assert lib.ft_attn_plan(None, 1, 1, 1, *z[:3]) == B.FT_ERR_INVALID_ARG
    assert lib.ft_attn_slots(None, 1, 1, 1, None, None, None, 8, *z[:9]) == B.FT_ERR_INVALID_ARG
    assert lib.ft_attn_forward(None, None, 0, None, None, 0, None, 0, None, 1.0, None) == B.FT_ERR_INVALID_ARG
    assert lib.ft_attn_sync_status(None) == B.FT_ERR_INVALID_ARG
    n = ctypes.c_uint64()
    assert lib.ft_attn_launch_count(None, ctypes.byref(n)) == B.FT_ERR_INVALID_ARG
