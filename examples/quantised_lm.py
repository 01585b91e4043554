"""N replicas of a small residual language model with 8-bit linear layers, trained by HDET on one GPU.

    python examples/quantised_lm.py [--steps 60]

The model predicts the next token from the current one: a fixed feature row of the token, then blocks of
    total = x + y_prev,   codes = root-mean-square norm of total in 8 bits,   y = codes W^T + b  (8-bit product),
then a last norm and an output layer with its cross-entropy in pieces of the vocabulary.  What a block keeps for its backward pass is its
8-bit input and the residual sum; weights are rounded to 8 bits at every step (the rounding counts as the identity in the gradients).
The gradients go into one plane a replica, which hdet_fanout_step applies at each replica's own rate; every T steps the replicas are
averaged and the controller moves the base rate.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_24708_amd as H  # noqa: E402

BF16 = torch.bfloat16


class Model:
    """Parameters, gradients and activations of `n` replicas: `blocks` blocks of width `d` over `vocab` tokens, `rows` tokens a step."""

    def __init__(self, n, blocks, d, vocab, rows, seed=0, device="cuda:0"):
        self.n, self.blocks, self.d, self.vocab, self.rows, self.device = n, blocks, d, vocab, rows, device
        g = torch.Generator(device=device).manual_seed(seed)
        shapes = []
        for b in range(blocks):
            shapes += [(f"gain{b}", (d,)), (f"w{b}", (d, d)), (f"b{b}", (d,))]
        shapes += [("gain", (d,)), ("head", (vocab, d)), ("head_b", (vocab,))]
        size = sum(-(-torch.Size(s).numel() // 4) * 4 for _, s in shapes)
        self.size = size
        self.stride = -(-size // 64) * 64
        self.params = torch.zeros(n, self.stride, device=device)
        self.grads = torch.zeros(n, self.stride, device=device)
        self.p, self.g, at = {}, {}, 0
        for name, s in shapes:
            k = torch.Size(s).numel()
            # views into the planes: [N, rows, columns] or [N, columns]
            self.p[name] = self.params[:, at:at + k].view(n, *s)
            self.g[name] = self.grads[:, at:at + k].view(n, *s)
            at += -(-k // 4) * 4
            if name.startswith("gain"):
                self.p[name].fill_(1.0)
            elif len(s) == 2:
                self.p[name].copy_(torch.randn(s, generator=g, device=device) * s[1] ** -0.5)      # every replica starts alike
        self.features = torch.randn(vocab, d, generator=g, device=device).to(BF16)

        def rows_of(dtype, width=d):
            return torch.empty(n, rows, width, dtype=dtype, device=device)

        def scalars():
            return torch.empty(n, rows, device=device)

        self.total = [rows_of(BF16) for _ in range(blocks + 1)]
        self.rstd = [scalars() for _ in range(blocks + 1)]
        self.codes = [H.hdet_codes_empty(n, rows, d, device) for _ in range(blocks)]
        self.scale = [scalars() for _ in range(blocks)]
        self.w_codes = [H.hdet_codes_empty(n, d, d, device) for _ in range(blocks)]
        self.w_scale = [torch.empty(n, d, device=device) for _ in range(blocks)]
        self.y, self.top = rows_of(BF16), rows_of(BF16)
        self.head = torch.empty(n, vocab, d, dtype=BF16, device=device)
        self.dy, self.dtotal = rows_of(BF16), rows_of(BF16)
        self.row_loss, self.loss = scalars(), torch.empty(n, device=device)
        bytes_ = max(H.hdet_vocab_loss_workspace(n, rows, d, vocab), H.hdet_rmsnorm_backward_workspace(n, rows, d),
                     H.hdet_quantised_linear_backward_workspace(n, rows, d, d))
        self.work = torch.empty(bytes_, dtype=torch.uint8, device=device)

    def forward_backward(self, ids, targets):
        """Losses [N] and, in self.grads, their gradients, for token ids and targets [N, rows]."""
        s = torch.cuda.current_stream().cuda_stream
        p, g, work = self.p, self.g, self.work
        x, y = self.features[ids], None
        for b in range(self.blocks):
            H.hdet_quantise_rows(p[f"w{b}"], self.w_codes[b], self.w_scale[b], stream=s)
            H.hdet_rmsnorm(x, p[f"gain{b}"], resid=y, total=self.total[b], codes=self.codes[b], scale=self.scale[b], rstd=self.rstd[b], stream=s)
            H.hdet_quantised_linear(self.codes[b], self.scale[b], self.w_codes[b], self.w_scale[b], self.y, bias=p[f"b{b}"], stream=s)
            x, y = self.total[b], self.y
        H.hdet_rmsnorm(x, p["gain"], resid=y, total=self.total[-1], y=self.top, rstd=self.rstd[-1], stream=s)
        self.head.copy_(p["head"])
        H.hdet_vocab_loss(self.top, self.head, targets, self.row_loss, self.loss, dh=self.dy, dw=g["head"], bias=p["head_b"], db=g["head_b"],
                          workspace=work, stream=s)
        # d(total) of the last norm is the gradient of both summands: of the stream below, and of the last block's y
        H.hdet_rmsnorm_backward(self.total[-1], p["gain"], self.rstd[-1], self.dy, self.dtotal, dgain=g["gain"], workspace=work, stream=s)
        for b in reversed(range(self.blocks)):
            H.hdet_quantised_linear_backward(self.dtotal, self.codes[b], self.scale[b], self.w_codes[b], self.w_scale[b], dx=self.dy, dw=g[f"w{b}"],
                                             db=g[f"b{b}"], workspace=work, stream=s)
            H.hdet_rmsnorm_backward(self.total[b], p[f"gain{b}"], self.rstd[b], self.dy, self.dtotal, dtotal=self.dtotal, dgain=g[f"gain{b}"],
                                    workspace=work, stream=s)
        return self.loss


def data(n, rows, vocab, seed, step, device):
    """Token ids and the next tokens of a fixed random successor table, one in eight replaced by noise, one in sixteen left out (-1)."""
    table = torch.randperm(vocab, generator=torch.Generator().manual_seed(seed))
    g = torch.Generator().manual_seed(seed * 1000003 + step)
    ids = torch.randint(0, vocab, (n, rows), generator=g)
    noise = torch.randint(0, vocab, (n, rows), generator=g)
    targets = torch.where(torch.rand(n, rows, generator=g) < 0.125, noise, table[ids])
    targets[torch.rand(n, rows, generator=g) < 0.0625] = -1
    return ids.to(device), targets.to(torch.int32).to(device)


def train(steps=60, n=4, blocks=2, d=128, vocab=1000, rows=512, sync=8, lr=3e-3, seed=0, device="cuda:0", show=print):
    """Losses [steps][N] of a run."""
    model = Model(n, blocks, d, vocab, rows, seed, device)
    # (a short run: the controller takes the rate over half way and lets it fall by a factor of 8, not of 250000)
    cfg = H.make_config(n_replicas=n, sync_interval=sync, total_steps=steps, warm_steps=steps // 2, lr_max=lr, f_div=1.0, f_final=8.0, constant_lr=1, alpha=0.2,
                        autolr_enabled=1, optimizer=H.HDET_ADAMW, weight_decay=0.01, model_kind=H.HDET_FLAT, n_params=model.size,
                        stream=torch.cuda.current_stream().cuda_stream)
    m, v = torch.zeros_like(model.params), torch.zeros_like(model.params)
    h = H.hdet_create(cfg, model.params, m, v, grads=model.grads, plane_stride=model.stride)
    losses, interval = [], torch.zeros(n, dtype=torch.float64)
    try:
        for t in range(1, steps + 1):
            ids, targets = data(n, rows, vocab, seed, t, device)
            step = model.forward_backward(ids, targets).double().cpu()
            H.hdet_fanout_step(h, None, H.HDET_FUSE_CONVERGE)
            losses.append(step.tolist())
            interval += step
            if t % sync == 0:
                H.hdet_converge(h)
                H.hdet_autolr_update(h, (interval / sync).tolist(), n)
                interval.zero_()
                show(f"step {t:4d}  losses " + " ".join(f"{x:.3f}" for x in losses[-1]))
    finally:
        torch.cuda.synchronize()
        H.hdet_destroy(h)
    return losses


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--steps", type=int, default=60)
    train(a.parse_args().steps)
