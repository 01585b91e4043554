"""hdet_attention with scales and caps at the ends of what it takes."""
import math

import pytest
import torch

import heads_reference as R
from test_lm_ops_attention import BF16, DEV, F32, forward, inputs, run_and_check

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


@each
@sizes
@pytest.mark.parametrize("scale,softcap", [(1e20, 1e-25), (-1e29, 1e-29), (1e10, 1e-10), (1e29, 1e5)])
def test_a_steep_cap(n, q_len, heads, d, dtype, scale, softcap):
    """scale / softcap beyond fp32: scores of 0 are 0, others the cap with their sign."""
    q, k, v, _ = inputs(n, 1, q_len, q_len, heads, heads, d, dtype, seed=d + 1)
    q.view(n, q_len, heads, d)[:, 1::2] = 0.0
    q.view(n, q_len, heads, d)[:, ::2, :, 1:] = 0.0
    k.view(n, q_len, heads, d)[..., 0] = torch.where(k.view(n, q_len, heads, d)[..., 0] < 0, -1.0, 1.0).to(dtype)
    q.view(n, q_len, heads, d)[:, ::2, :, 0] = 1.0
    out, lse = forward(q, k, v, heads, heads, 1, scale=scale, softcap=softcap, causal=False)
    sign = math.copysign(1.0, scale) * k.view(n, q_len, heads, d)[..., 0].double().transpose(1, 2)[:, :, None]       # [n, heads, 1, keys]
    z = torch.zeros(n, heads, q_len, q_len, dtype=torch.float64, device=DEV)
    z[:, :, ::2] = softcap * sign
    want_lse = torch.logsumexp(z, -1)
    p = torch.exp(z - want_lse[..., None])
    vh = v.double().view(n, q_len, heads, d).transpose(1, 2).contiguous()
    want, size = (torch.matmul(p, x).transpose(1, 2).reshape(n, q_len, heads * d) for x in (vh, vh.abs()))
    # scores off by 4 steps of the cap and 16 of one; p as R.attention has it
    off = R.U * (4.0 * softcap + 16.0)
    R.check(lse, want_lse, (off + R.U * (q_len + 24) + R.U * want_lse.abs()), "lse")
    b = R.half(dtype)
    R.check(out, want, (2.0 * off + 4.0 * R.U * (softcap + 8.0) + R.U * (q_len + 16) + (b if dtype == BF16 else 0.0)) * size + b * want.abs(), "out")
