"""hdet_attention on values at the upper end of their type: a mean of numbers of the type is one."""
import pytest
import torch

import heads_reference as R
from test_lm_ops_attention import BF16, DEV, F32, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,q_len,kv_len,heads,d", [(16, 300, 600, 16, 64), (16, 300, 1700, 16, 128), (8, 1, 5000, 4, 64), (1, 1, 40000, 2, 128), (16, 300, 600, 16, 40), (1, 3, 70, 1, 1)])
@pytest.mark.parametrize("how", [dict(causal=False), dict(causal=True, window=200), dict(causal=False, softcap=3.0)], ids=str)
def test_values_near_the_largest(n, q_len, kv_len, heads, d, how, dtype):
    """Columns from 10^30 to 3 x 10^38 and ordinary ones next to them, in some blocks only; a maximum that comes late."""
    q, k, v, _ = inputs(n, 1, q_len, kv_len, heads, heads, d, dtype, seed=d + kv_len)
    columns = v.view(n, kv_len, heads, d)
    columns[..., 0] = columns[..., 0].abs().clamp(max=2.5).to(dtype) * 1e38
    if d > 9:
        columns[..., 9] *= 1e37
        columns[..., 7] *= 1e30
    k.view(n, kv_len, heads, d)[:, kv_len // 2:] *= 4
    out, lse = forward(q, k, v, heads, heads, 1, **how)
    want = R.attention(q, k, v, heads, heads, 1, **how)
    R.check(out, want["out"], want["bound_out"], "out")
    R.check(lse, want["lse"], want["bound_lse"], "lse")
