"""N replicas of a small language model with attention over packed documents, trained by HDET on one GPU.

    python examples/attention_lm.py [--steps 60]

Rows are `seqs` sequences of tokens a replica, each a few documents behind each other and some padding; a token attends the tokens of its own document up to itself.
A block is
    total = x + y_prev,   codes = root-mean-square norm of total in 8 bits,   q | k | v = codes W^T + b  (8-bit product),
    q, k = heads normed and rotated by the position in the document,   a = attention,   y = (a in 8 bits) W_o^T + b_o
and behind the blocks come a last norm and an output layer with its cross-entropy.  Gradients are formed in tensors of their own; their common norm bounds them on
their way into the plane that hdet_fanout_step applies at each replica's rate.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_24708_amd as H  # noqa: E402

BF16 = torch.bfloat16


class Model:
    """Parameters, gradients and activations of `n` replicas: `blocks` blocks of `heads` query and `kv_heads` key heads of `head_dim` columns over `vocab` tokens."""

    def __init__(self, n, blocks, heads, kv_heads, head_dim, vocab, seqs, length, softcap=30.0, max_norm=1.0, seed=0, device="cuda:0"):
        d, self.wide = heads * head_dim, (heads + 2 * kv_heads) * head_dim
        rows = seqs * length
        self.n, self.blocks, self.heads, self.kv_heads, self.head_dim, self.d = n, blocks, heads, kv_heads, head_dim, d
        self.vocab, self.seqs, self.length, self.rows, self.softcap, self.max_norm, self.device = vocab, seqs, length, rows, softcap, max_norm, device
        g = torch.Generator(device=device).manual_seed(seed)
        shapes = []
        for b in range(blocks):
            shapes += [(f"gain{b}", (d,)), (f"qkv{b}", (self.wide, d)), (f"qkv_b{b}", (self.wide,)), (f"q_gain{b}", (head_dim,)), (f"k_gain{b}", (head_dim,)),
                       (f"o{b}", (d, d)), (f"o_b{b}", (d,))]
        shapes += [("gain", (d,)), ("head", (vocab, d)), ("head_b", (vocab,))]
        self.size = sum(-(-torch.Size(s).numel() // 4) * 4 for _, s in shapes)
        self.stride = -(-self.size // 64) * 64
        self.params = torch.zeros(n, self.stride, device=device)
        self.grads = torch.zeros(n, self.stride, device=device)          # the bounded gradients, as the update takes them
        self.p, self.g, outs, at = {}, {}, [], 0
        for name, s in shapes:
            k = torch.Size(s).numel()
            self.p[name] = self.params[:, at:at + k].view(n, *s)
            self.g[name] = torch.zeros(n, *s, device=device)
            outs.append(self.grads[:, at:at + k].view(n, *s))
            at += -(-k // 4) * 4
            if "gain" in name:
                self.p[name].fill_(1.0)
            elif len(s) == 2:
                self.p[name].copy_(torch.randn(s, generator=g, device=device) * s[1] ** -0.5)
        self.list = H.hdet_gradient_list(list(self.g.values()), outs)
        self.features = torch.randn(vocab, d, generator=g, device=device).to(BF16)
        self.freq = H.hdet_rotary_frequencies(head_dim, device=device)

        def rows_of(width, dtype=BF16):
            return torch.empty(n, rows, width, dtype=dtype, device=device)

        def scalars(count=rows):
            return torch.empty(n, count, device=device)

        each = range(blocks)
        self.total, self.rstd = [rows_of(d) for _ in range(blocks + 1)], [scalars() for _ in range(blocks + 1)]
        self.codes, self.scale = [H.hdet_codes_empty(n, rows, d, device) for _ in each], [scalars() for _ in each]
        self.a_codes, self.a_scale = [H.hdet_codes_empty(n, rows, d, device) for _ in each], [scalars() for _ in each]
        self.w_codes, self.w_scale = [H.hdet_codes_empty(n, self.wide, d, device) for _ in each], [scalars(self.wide) for _ in each]
        self.o_codes, self.o_scale = [H.hdet_codes_empty(n, d, d, device) for _ in each], [scalars(d) for _ in each]
        self.qkv, self.turned = [rows_of(self.wide) for _ in each], [rows_of((heads + kv_heads) * head_dim) for _ in each]
        self.a, self.lse = [rows_of(d) for _ in each], [torch.empty(n, heads, rows, device=device) for _ in each]
        self.y, self.top, self.dy, self.da, self.dtotal, self.dqkv = rows_of(d), rows_of(d), rows_of(d), rows_of(d), rows_of(d), rows_of(self.wide)
        self.head = torch.empty(n, vocab, d, dtype=BF16, device=device)
        self.row_loss, self.loss, self.norm = scalars(), torch.empty(n, device=device), torch.empty(n, device=device)
        self.sizes = (n, seqs, length, length, heads, kv_heads, head_dim)
        bytes_ = max(H.hdet_vocab_loss_workspace(n, rows, d, vocab), H.hdet_rmsnorm_backward_workspace(n, rows, d),
                     H.hdet_quantised_linear_backward_workspace(n, rows, d, self.wide), H.hdet_quantised_linear_backward_workspace(n, rows, d, d),
                     H.hdet_head_rotary_backward_workspace(n, rows, head_dim, heads, kv_heads), H.hdet_attention_workspace(*self.sizes),
                     H.hdet_attention_backward_workspace(*self.sizes), H.hdet_clip_gradients_workspace(n, len(self.list)))
        self.work = torch.empty(bytes_, dtype=torch.uint8, device=device)

    def forward_backward(self, ids, targets, first, end, positions):
        """Losses [N] and, in self.grads, their bounded gradients, for token ids and targets [N, rows]; first, end: the keys that each token attends, positions: its place in its
        document (int32 [N, rows])."""
        s = torch.cuda.current_stream().cuda_stream
        p, g, work, hd = self.p, self.g, self.work, self.head_dim
        at, cut = self.heads * hd, (self.heads + self.kv_heads) * hd
        mask = dict(causal=False, softcap=self.softcap, first=first, end=end, stream=s)
        turn = dict(freq=self.freq, positions=positions, stream=s)
        x, y = self.features[ids], None
        for b in range(self.blocks):
            H.hdet_quantise_rows(p[f"qkv{b}"], self.w_codes[b], self.w_scale[b], stream=s)
            H.hdet_quantise_rows(p[f"o{b}"], self.o_codes[b], self.o_scale[b], stream=s)
            H.hdet_rmsnorm(x, p[f"gain{b}"], resid=y, total=self.total[b], codes=self.codes[b], scale=self.scale[b], rstd=self.rstd[b], stream=s)
            qkv, t = self.qkv[b], self.turned[b]
            H.hdet_quantised_linear(self.codes[b], self.scale[b], self.w_codes[b], self.w_scale[b], qkv, bias=p[f"qkv_b{b}"], stream=s)
            H.hdet_head_rotary(qkv[..., :at], t[..., :at], hd, k=qkv[..., at:cut], k_out=t[..., at:], q_gain=p[f"q_gain{b}"], k_gain=p[f"k_gain{b}"], **turn)
            H.hdet_attention(t[..., :at], t[..., at:], qkv[..., cut:], self.a[b], self.heads, self.kv_heads, self.seqs, lse=self.lse[b], workspace=work, **mask)
            H.hdet_quantise_rows(self.a[b], self.a_codes[b], self.a_scale[b], stream=s)
            H.hdet_quantised_linear(self.a_codes[b], self.a_scale[b], self.o_codes[b], self.o_scale[b], self.y, bias=p[f"o_b{b}"], stream=s)
            x, y = self.total[b], self.y
        H.hdet_rmsnorm(x, p["gain"], resid=y, total=self.total[-1], y=self.top, rstd=self.rstd[-1], stream=s)
        self.head.copy_(p["head"])
        H.hdet_vocab_loss(self.top, self.head, targets, self.row_loss, self.loss, dh=self.dy, dw=g["head"], bias=p["head_b"], db=g["head_b"], workspace=work, stream=s)
        H.hdet_rmsnorm_backward(self.total[-1], p["gain"], self.rstd[-1], self.dy, self.dtotal, dgain=g["gain"], workspace=work, stream=s)
        for b in reversed(range(self.blocks)):
            qkv, t, d3 = self.qkv[b], self.turned[b], self.dqkv
            H.hdet_quantised_linear_backward(self.dtotal, self.a_codes[b], self.a_scale[b], self.o_codes[b], self.o_scale[b], dx=self.da, dw=g[f"o{b}"], db=g[f"o_b{b}"],
                                             workspace=work, stream=s)
            H.hdet_attention_backward(t[..., :at], t[..., at:], qkv[..., cut:], self.a[b], self.lse[b], self.da, d3[..., :at], d3[..., at:cut], d3[..., cut:], self.heads,
                                      self.kv_heads, self.seqs, workspace=work, **mask)
            H.hdet_head_rotary_backward(qkv[..., :at], d3[..., :at], d3[..., :at], hd, k=qkv[..., at:cut], dk_out=d3[..., at:cut], dk=d3[..., at:cut],
                                        q_gain=p[f"q_gain{b}"], k_gain=p[f"k_gain{b}"], dq_gain=g[f"q_gain{b}"], dk_gain=g[f"k_gain{b}"], workspace=work, **turn)
            H.hdet_quantised_linear_backward(d3, self.codes[b], self.scale[b], self.w_codes[b], self.w_scale[b], dx=self.dy, dw=g[f"qkv{b}"], db=g[f"qkv_b{b}"],
                                             workspace=work, stream=s)
            H.hdet_rmsnorm_backward(self.total[b], p[f"gain{b}"], self.rstd[b], self.dy, self.dtotal, dtotal=self.dtotal, dgain=g[f"gain{b}"], workspace=work, stream=s)
        H.hdet_clip_gradients(self.list, self.norm, self.max_norm, workspace=work, stream=s)
        return self.loss


def data(n, seqs, length, vocab, seed, step, device):
    """Token ids, targets (-1 behind the last document), first and end keys and positions.  A document repeats a random word of 4 to 9 tokens, so that what follows
    a token is to be read off its earlier occurrence."""
    g = torch.Generator().manual_seed(seed * 1000003 + step)
    ids, targets = torch.zeros(n * seqs, length, dtype=torch.int64), torch.full((n * seqs, length), -1, dtype=torch.int32)
    first, end, pos = (torch.zeros(n * seqs, length, dtype=torch.int32) for _ in range(3))
    for s in range(n * seqs):
        at, last = 0, length - int(torch.randint(0, length // 8 + 1, (1,), generator=g))
        while at < last:
            stop = min(last, at + int(torch.randint(length // 4, length // 2, (1,), generator=g)))
            word = torch.randint(0, vocab, (int(torch.randint(4, 10, (1,), generator=g)),), generator=g)
            text = word.repeat(-(-(stop - at + 1) // len(word)))[:stop - at + 1]
            here = torch.arange(stop - at, dtype=torch.int32)
            ids[s, at:stop], targets[s, at:stop] = text[:-1], text[1:].to(torch.int32)
            first[s, at:stop], end[s, at:stop], pos[s, at:stop] = at, at + here + 1, here
            at = stop
    return [x.view(n, seqs * length).to(device) for x in (ids, targets, first, end, pos)]


def train(steps=60, n=4, blocks=2, heads=4, kv_heads=2, head_dim=32, vocab=200, seqs=4, length=128, sync=8, lr=3e-3, seed=0, device="cuda:0", show=print):
    """Losses [steps][N] of a run."""
    model = Model(n, blocks, heads, kv_heads, head_dim, vocab, seqs, length, seed=seed, device=device)
    cfg = H.make_config(n_replicas=n, sync_interval=sync, total_steps=steps, warm_steps=steps // 2, lr_max=lr, f_div=1.0, f_final=8.0, constant_lr=1, alpha=0.2,
                        autolr_enabled=1, optimizer=H.HDET_ADAMW, weight_decay=0.01, model_kind=H.HDET_FLAT, n_params=model.size,
                        stream=torch.cuda.current_stream().cuda_stream)
    m, v = torch.zeros_like(model.params), torch.zeros_like(model.params)
    h = H.hdet_create(cfg, model.params, m, v, grads=model.grads, plane_stride=model.stride)
    losses, interval = [], torch.zeros(n, dtype=torch.float64)
    try:
        for t in range(1, steps + 1):
            step = model.forward_backward(*data(n, seqs, length, vocab, seed, t, device)).double().cpu()
            H.hdet_fanout_step(h, None, H.HDET_FUSE_CONVERGE)
            losses.append(step.tolist())
            interval += step
            if t % sync == 0:
                H.hdet_converge(h)
                H.hdet_autolr_update(h, (interval / sync).tolist(), n)
                interval.zero_()
                show(f"step {t:4d}  losses " + " ".join(f"{x:.3f}" for x in losses[-1]) + "  norms " + " ".join(f"{x:.2f}" for x in model.norm.tolist()))
    finally:
        torch.cuda.synchronize()
        H.hdet_destroy(h)
    return losses


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--steps", type=int, default=60)
    train(a.parse_args().steps)
