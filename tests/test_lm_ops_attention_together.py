"""Rotated heads, attention and clipped gradients with the other language-model operators: the example's model against 64-bit automatic differentiation, a training run,
and the clipped gradient between hdet_forward_backward and hdet_fanout_step."""
import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import heads_reference as R  # noqa: E402
import ops_reference as O  # noqa: E402
import paper_2604_24708_amd as H  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Through(torch.autograd.Function):
    """Rows to 8 bits and back, with the identity as its gradient."""

    @staticmethod
    def forward(ctx, v):
        q, s = O.rows8(v)
        return q * s

    @staticmethod
    def backward(ctx, g):
        return g


def norm(u, gain, eps):
    return u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps) * gain


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 2, 16), (2, 1, 40)])
def test_a_step_against_automatic_differentiation(heads, kv_heads, head_dim):
    """Activations and their gradients are rounded to bfloat16 at about a dozen places on the way through a block (2^-9 each in the mean), inputs to 8 bits at two, and codes that fall the other
    way for it: whole tensors agree to a few per cent; a missing term would be off by the tensor's size."""
    import attention_lm as E
    n, blocks, vocab, seqs, length = 2, 2, 97, 3, 60
    model = E.Model(n, blocks, heads, kv_heads, head_dim, vocab, seqs, length, softcap=5.0, max_norm=0.25, seed=3)
    ids, targets, first, end, pos = E.data(n, seqs, length, vocab, 5, 1, DEV)
    model.params[1] += 0.05 * torch.randn(model.params[1].shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    loss = model.forward_backward(ids, targets, first, end, pos).clone()
    leaves = {k: v.detach().double().clone().requires_grad_(True) for k, v in model.p.items()}
    rows, d = seqs * length, heads * head_dim
    at, cut, group = heads * head_dim, (heads + kv_heads) * head_dim, heads // kv_heads
    j = torch.arange(length, device=DEV)
    seen = ((j >= first.view(n, seqs, length, 1)) & (j < end.view(n, seqs, length, 1)))[:, :, None]
    freq = R.frequencies(head_dim)

    def split(x, count):
        return x.view(n, seqs, length, count, head_dim).transpose(2, 3)

    x = model.features[ids].double()
    total = x
    for b in range(blocks):
        codes = Through.apply(norm(total, leaves[f"gain{b}"][:, None], 1e-5))
        qkv = torch.matmul(codes, Through.apply(leaves[f"qkv{b}"]).transpose(1, 2)) + leaves[f"qkv_b{b}"][:, None]
        q, k = (R.turn(norm(t.view(n, rows, -1, head_dim), leaves[name + str(b)][:, None, None], 1e-6), pos, freq, False, 1.0).reshape(n, rows, -1)
                for t, name in ((qkv[..., :at], "q_gain"), (qkv[..., at:cut], "k_gain")))
        q, k, v = split(q, heads), split(k, kv_heads).repeat_interleave(group, 2), split(qkv[..., cut:], kv_heads).repeat_interleave(group, 2)
        z = 5.0 * torch.tanh(torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(head_dim) / 5.0)
        p = torch.softmax(z.masked_fill(~seen, -1e30), -1).masked_fill(~seen, 0.0)
        a = torch.matmul(p, v).transpose(2, 3).reshape(n, rows, d)
        total = total + torch.matmul(Through.apply(a), Through.apply(leaves[f"o{b}"]).transpose(1, 2)) + leaves[f"o_b{b}"][:, None]
    z = torch.matmul(norm(total, leaves["gain"][:, None], 1e-5), leaves["head"].transpose(1, 2)) + leaves["head_b"][:, None]
    ok = targets >= 0
    mean = ((torch.logsumexp(z, -1) - z.gather(-1, targets.long().clamp(min=0)[..., None])[..., 0]) * ok).sum(-1) / ok.sum(-1)
    mean.sum().backward()
    assert torch.all((loss.double() - mean).abs() <= 2.0 ** -6 * mean.abs())
    for k, v in leaves.items():
        if k.startswith("qkv_b"):
            # a bias of all keys of a row moves all its scores alike but for the norm, the rotation and the cap: held to the gradient of the whole layer
            assert float((model.g[k].double() - v.grad).norm()) <= 0.05 * float(leaves["qkv" + k[5:]].grad.norm()), k
        else:
            assert O.rel(model.g[k], v.grad) <= 0.08, k
    # the plane holds them, bounded by their common norm
    size = torch.sqrt(sum(g.double().reshape(n, -1).square().sum(1) for g in model.g.values()))
    assert bool((size > 0.25).all())
    R.check(model.norm, size, 2 * R.U * size, "norm")
    spot = 0
    for name, g in model.g.items():
        k = g[0].numel()
        want = g.double().reshape(n, -1) * (0.25 / size)[:, None]
        R.check(model.grads[:, spot:spot + k], want, 4 * R.U * want.abs() + 2.0 ** -149, name)
        spot += -(-k // 4) * 4


def test_a_training_run():
    import attention_lm as E
    losses = np.array(E.train(steps=24, n=3, blocks=1, heads=2, kv_heads=1, head_dim=32, vocab=50, seqs=2, length=64, sync=8, show=lambda *_: None))
    assert losses.shape == (24, 3) and np.isfinite(losses).all()
    again = np.array(E.train(steps=24, n=3, blocks=1, heads=2, kv_heads=1, head_dim=32, vocab=50, seqs=2, length=64, sync=8, show=lambda *_: None))
    assert (losses == again).all()


def test_clipped_gradients_of_a_model():
    """hdet_forward_backward, the bound on its gradient planes, hdet_fanout_step: the update of the bounded gradient."""
    import hdet_inputs as I
    from harness import library_config
    from oracle import hdet_oracle as T
    n, cfg = 2, dict(n_blocks=1, d_model=16, n_heads=2, d_ff=32, seq_len=8, vocab=31)
    size = I.transformer_param_count(cfg)
    stride = (size + 63) // 64 * 64
    d = dict(n_replicas=n, total_steps=4, sync_interval=4, warm_steps=4, lr_max=0.5, alpha=0.2, autolr_enabled=False, optimizer=T.SGDM, momentum=0.0, weight_decay=0.0,
             grad_mode=T.GRAD_PER_REPLICA, seed=7)
    host = np.zeros((n, stride), np.float32)
    host[:, :size] = I.transformer_init(n, cfg, I.SEED_INIT, std=0.1, bias_std=0.05)
    theta = torch.from_numpy(host).to(DEV)
    m, g = torch.zeros_like(theta), torch.zeros_like(theta)
    lc = library_config(d, model_kind=H.HDET_TRANSFORMER, batch=2, precision=H.HDET_FP32, **cfg)
    ws = torch.empty(H.hdet_workspace_bytes(lc, stride)[2], dtype=torch.uint8, device=DEV)
    h = H.hdet_create(lc, theta, m, None, grads=g, workspace=ws, plane_stride=stride)
    try:
        ids, tgt = I.zipf_tokens(n, 2, cfg["seq_len"], cfg["vocab"], I.SEED_DATA, 1)
        H.hdet_forward_backward(h, torch.from_numpy(ids).to(DEV), torch.from_numpy(tgt).to(DEV))
        whole = g.double()
        places, at = [], 0
        for _, s in I.transformer_shapes(cfg):
            k = int(np.prod(s))
            places.append(g[:, at:at + k])
            at += k
        assert at == size
        norm_, work = torch.empty(n, device=DEV), torch.empty(H.hdet_clip_gradients_workspace(n, len(places)), dtype=torch.uint8, device=DEV)
        before = theta.double()
        H.hdet_clip_gradients(H.hdet_gradient_list(places), norm_, 0.01, workspace=work)
        H.hdet_fanout_step(h, None, 0)
        norms = whole[:, :size].norm(dim=1)
        assert bool((norms > 0.01).all())
        R.check(norm_, norms, 2 * R.U * norms, "norm")
        rates = torch.tensor(list(H.hdet_get_state(h).lr)[:n], device=DEV, dtype=torch.float64)
        want = before - rates[:, None] * whole * (0.01 / norms)[:, None]
        R.check(theta, want, 8 * R.U * (before.abs() + (before - want).abs()) + 1e-12, "parameters")
    finally:
        torch.cuda.synchronize()
        H.hdet_destroy(h)
