"""GPU tests of the attention operators at their edges: windows, infinities and NaN, entries that cannot be, empty steps, long
prompts, many work items, replay from a graph."""
import numpy as np
import pytest
import torch

from paper_2608_16157_b200 import attention as A
from paper_2608_16157_b200 import binding as B
from tests import attn_reference as R
from tests.test_gpu_attn import DEV, i32, make_attn, run_attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 30, 1 << 30])
def test_a_window_wider_than_any_request_is_no_window(window):
    """Also for requests whose first rows stand before position 0 (more new rows than cached tokens)."""
    run_attn("bf16", 8, 2, 128, 16, window, [(1, 0), (40, 13), (2, 1), (30, 3), (60, 300), (1, 70)], seed=1)
    run_attn("fp16", 16, 2, 64, 32, window, [(40, 13), (300, 7), (0, 9), (2, 100)], seed=2)
