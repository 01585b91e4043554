"""The rotation's outputs and gradients, and the clipped gradient, in the places of their inputs: the same bits as next to them."""
import pytest
import torch

import heads_reference as R
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
each = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


@each
@pytest.mark.parametrize("paired", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("n,rows,heads,k_heads,d,rotated", [(2, 300, 8, 2, 64, 64), (3, 77, 5, 1, 50, 18), (1, 2000, 4, 4, 128, 64), (2, 33, 3, 3, 7, 6)])
@pytest.mark.parametrize("over", ["dq_out", "q", "one of each"])
def test_rotation(n, rows, heads, k_heads, d, rotated, paired, over, dtype):
    """q | k are columns of one matrix, and so are their outputs, the gradients there, and the gradients."""
    wide, at = (heads + k_heads) * d, heads * d
    qk, dy = (normal(s, n, rows, wide).to(dtype) for s in (1, 2))
    gains = [normal(3, n, d), normal(4, n, d)]
    how = dict(q_gain=gains[0], k_gain=gains[1], freq=R.frequencies(rotated), paired=paired, eps=1e-6)
    y, dx = torch.empty_like(qk), torch.empty_like(qk)
    work = torch.zeros(H.hdet_head_rotary_backward_workspace(n, rows, d, heads, k_heads), dtype=torch.uint8, device=DEV)

    def backward(x, g, q_to, k_to):
        dgain = [torch.empty_like(gains[0]) for _ in range(2)]
        H.hdet_head_rotary_backward(x[..., :at], g[..., :at], q_to[..., :at], d, k=x[..., at:], dk_out=g[..., at:], dk=k_to[..., at:], dq_gain=dgain[0], dk_gain=dgain[1], workspace=work, **how)
        return dgain

    want_gain = backward(qk, dy, dx, dx)
    H.hdet_head_rotary(qk[..., :at], y[..., :at], d, k=qk[..., at:], k_out=y[..., at:], **how)
    x, g = qk.clone(), dy.clone()
    q_to, k_to = {"dq_out": (g, g), "q": (x, x), "one of each": (x, g)}[over]
    got_gain = backward(x, g, q_to, k_to)
    assert torch.equal(q_to[..., :at], dx[..., :at]) and torch.equal(k_to[..., at:], dx[..., at:])
    assert all(torch.equal(a, b) for a, b in zip(got_gain, want_gain))
    x = qk.clone()
    H.hdet_head_rotary(x[..., :at], x[..., :at], d, k=x[..., at:], k_out=x[..., at:], **how)
    assert torch.equal(x, y)


@pytest.mark.parametrize("shared", [False, True], ids=["own", "shared"])
@pytest.mark.parametrize("shape,pitch", [((3,), 3), ((100, 333), 333), ((100, 333), 340), ((257, 1024), 1024), ((1, 8193), 8200)])
def test_clipped_gradients(shape, pitch, shared):
    """An fp32 output that is its gradient, strides and all."""
    n = 3
    full = normal(5, n, *shape[:-1], pitch)
    g = full[..., : shape[-1]]
    out, norm, norm2 = torch.empty(n, *shape, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    work = torch.zeros(H.hdet_clip_gradients_workspace(n, 1), dtype=torch.uint8, device=DEV)
    H.hdet_clip_gradients(H.hdet_gradient_list([g], [out]), norm, 0.5, shared=shared, workspace=work)
    before = full.clone()
    H.hdet_clip_gradients(H.hdet_gradient_list([g], [g]), norm2, 0.5, shared=shared, workspace=work)
    assert torch.equal(g, out) and torch.equal(norm, norm2) and bool((norm > 0.5).all())
    assert torch.equal(full[..., shape[-1]:], before[..., shape[-1]:])
