"""hdet_attention with scales at the ends of what it takes."""
import pytest

from test_lm_ops_attention import BF16, F32, inputs, run_and_check

pytestmark = pytest.mark.gpu
each = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
# few queries and blocks of 128 of them
sizes = pytest.mark.parametrize("n,q_len,heads,d", [(1, 70, 2, 64), (16, 300, 16, 64), (16, 300, 16, 128), (2, 70, 2, 40)])


@each
@sizes
@pytest.mark.parametrize("scale", [1e-300, 1e-46, 1e-45, 1e-40, -1e-46, 1e-30])
def test_scales_below_fp32(n, q_len, heads, d, dtype, scale):
    """Scores of nearly 0 under a causal mask: the mean of the values so far; the gradients at queries and keys are as small as the scale."""
    q, k, v, dout = inputs(n, 1, q_len, q_len, heads, heads, d, dtype, seed=d)
    run_and_check(q, k, v, dout, heads, heads, 1, scale=scale)
