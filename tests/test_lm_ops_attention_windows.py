"""Gradients of windowed attention where dk and dv in fp32 are made by several launches that add up: windows around multiples of a tile and of a launch's 1024 rows, groups, odd offsets of the
queries against the keys, ranges that the window does not bound."""
import pytest
import torch

from test_lm_ops_attention import BF16, F32, inputs, ints, run_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 33, 64, 129, 130, 161, 895, 896, 897, 898, 929, 1000])
def test_windows(window, dtype):
    """Whole walks: blocks enough.  A group of two heads: 1024 rows are 512 queries of each."""
    q, k, v, dout = inputs(20, 1, 1100, 1100, 16, 8, 16, dtype, seed=window)
    run_and_check(q[:1], k[:1], v[:1], dout[:1], 16, 8, 1, window=window)
    n = 20 if window in (33, 897) else 4
    run_and_check(q[:n], k[:n], v[:n], dout[:n], 16, 8, 1, window=window)


@pytest.mark.parametrize("q_len,kv_len", [(1500, 1337), (1337, 1500), (2100, 2100)])
@pytest.mark.parametrize("heads,kv_heads,d", [(8, 1, 64), (4, 4, 72)])
def test_other_lengths_and_masks(q_len, kv_len, heads, kv_heads, d):
    q, k, v, dout = inputs(1, 1, q_len, kv_len, heads, kv_heads, d, F32, seed=q_len)
    for window in (200, 1030):
        run_and_check(q, k, v, dout, heads, kv_heads, 1, window=window)
        run_and_check(q, k, v, dout, heads, kv_heads, 1, window=window, causal=False)
        # every query at one of a few positions: the window says nothing about how many queries see a key
        positions = ints(torch.randint(0, 40, (1, q_len), generator=torch.Generator().manual_seed(3)))
        run_and_check(q, k, v, dout, heads, kv_heads, 1, window=window, positions=positions)
