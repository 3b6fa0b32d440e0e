"""The limits of the attention operators' configuration, as their header states them."""
import pytest

from paper_2608_16157_b200 import attention as A

GOOD = dict(n_q_heads=32, n_kv_heads=4, head_dim=128, page_tokens=16, n_pages=64, max_requests=8, max_tokens=64, max_pages=8)


@pytest.mark.parametrize("inside,beyond", [
    (dict(n_pages=(1 << 22) - 1), dict(n_pages=1 << 22)),
    (dict(n_pages=(1 << 22) - 1, page_tokens=128, max_pages=(1 << 24) - 1, max_requests=1, n_kv_heads=4, n_q_heads=4),
     dict(n_pages=(1 << 22) - 1, page_tokens=128, max_pages=1 << 24, max_requests=1, n_kv_heads=4, n_q_heads=4)),
    (dict(n_q_heads=1024, n_kv_heads=16), dict(n_q_heads=1025, n_kv_heads=25)),
    (dict(n_q_heads=256), dict(n_q_heads=260)),
    (dict(max_requests=1024), dict(max_requests=1025)),
    (dict(max_tokens=1 << 20), dict(max_tokens=(1 << 20) + 1)),
    (dict(max_requests=128, max_pages=1 << 23), dict(max_requests=128, max_pages=1 << 24)),           # work units: 2^22 blocks x 4 heads x 128
    (dict(max_tokens=1 << 20, max_pages=1 << 15), dict(max_tokens=1 << 20, max_pages=1 << 16)),       # 2^14 blocks x 4 heads x 2^15 pieces
])
def test_limits(inside, beyond):
    assert A.cache_bytes(A.make_config(**{**GOOD, **inside})) > 0
    assert A.cache_bytes(A.make_config(**{**GOOD, **beyond})) == 0
