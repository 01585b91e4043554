"""The language-model operators together: the example's model against 64-bit automatic differentiation, and a short training run."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import ops_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu


class Through(torch.autograd.Function):
    """Rows to 8 bits and back, with the identity as its gradient."""

    @staticmethod
    def forward(ctx, v):
        q, s = R.rows8(v)
        return q * s

    @staticmethod
    def backward(ctx, g):
        return g


def test_a_step_against_automatic_differentiation():
    """Activations and their gradients are rounded to bfloat16 at half a dozen places on the way (2^-9 each in the mean, and a code that falls the other way for it), so
    whole tensors agree to a few times 2^-9 times the depth; a missing term would be off by the tensor's size."""
    import quantised_lm as E
    n, blocks, d, vocab, rows = 2, 2, 72, 301, 160
    model = E.Model(n, blocks, d, vocab, rows, seed=3)
    ids, targets = E.data(n, rows, vocab, 5, 1, "cuda:0")
    model.params[1] += 0.05 * torch.randn(model.params[1].shape, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(1))
    loss = model.forward_backward(ids, targets).clone()
    leaves = {k: v.detach().double().clone().requires_grad_(True) for k, v in model.p.items()}

    def norm(u, gain):
        return u / torch.sqrt((u * u).mean(-1, keepdim=True) + 1e-5) * gain[:, None]

    x = model.features[ids].double()
    total = x
    for b in range(blocks):
        codes = Through.apply(norm(total, leaves[f"gain{b}"]))
        y = torch.matmul(codes, Through.apply(leaves[f"w{b}"]).transpose(1, 2)) + leaves[f"b{b}"][:, None]
        total = total + y
    top = norm(total, leaves["gain"])
    head = leaves["head"]
    z = torch.matmul(top, head.transpose(1, 2)) + leaves["head_b"][:, None]
    ok = targets >= 0
    lse = torch.logsumexp(z, -1) - z.gather(-1, targets.long().clamp(min=0)[..., None])[..., 0]
    mean = (lse * ok).sum(-1) / ok.sum(-1)
    mean.sum().backward()
    assert torch.all((loss.double() - mean).abs() <= 2.0 ** -7 * mean.abs())
    for k, v in leaves.items():
        assert R.rel(model.g[k], v.grad) <= 0.05, k


def test_training_lowers_the_loss_of_every_replica():
    import quantised_lm as E
    losses = E.train(steps=48, n=3, blocks=2, d=64, vocab=200, rows=256, sync=8, lr=5e-3, show=lambda *_: None)
    first, last = torch.tensor(losses[:4]).mean(0), torch.tensor(losses[-4:]).mean(0)
    assert torch.all(last < 0.6 * first), (first, last)
