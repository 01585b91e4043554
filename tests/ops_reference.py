"""Language-model operators in 64 bits, from their formulas, and the error bounds that the tests of the kernels hold them to.

A sum of K terms formed in fp32 in any order is off by at most about depth * 2^-24 times the sum of the terms' sizes, depth being the longest chain
of additions a term goes through; U below is 2^-24.  A result rounded to bfloat16 is off by half a unit in its eighth bit: at most 2^-8 of itself.
"""
import torch

U = 2.0 ** -24
DEV = "cuda:0"


def half_ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def scale_exponent(top):
    """The smallest e >= -126 with top <= 127 * 2^e (top: fp64, finite)."""
    e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -140) / 127.0))
    e = torch.where(127.0 * torch.exp2(e) < top, e + 1, e)
    e = torch.where(127.0 * torch.exp2(e - 1) >= top, e - 1, e)
    return torch.clamp(e, min=-126.0)


def rows8(v):
    """Codes (fp64) and scales (fp64) of the rows of v (fp64)."""
    s = torch.exp2(scale_exponent(v.abs().amax(-1, keepdim=True)))
    return torch.round(v / s), s


def norm(x, resid, gain, eps):
    u = x.double() + (0.0 if resid is None else resid.double())
    rstd = 1.0 / torch.sqrt((u * u).mean(-1) + eps)
    return u, rstd, u * rstd[..., None] * gain.double()[:, None]


def norm_backward(total, gain, rstd, dy, dtotal):
    h, r, g, d = total.double(), rstd.double()[..., None], gain.double()[:, None], dy.double()
    xh, dn = h * r, d * g
    dx = r * (dn - xh * (dn * xh).mean(-1, keepdim=True)) + (0.0 if dtotal is None else dtotal.double())
    return dx, (d * xh).sum(1)


def vocab_loss(h, w, bias, labels):
    """row losses, means, dh, dw, db and dz (all fp64)."""
    z = torch.matmul(h.double(), w.double().transpose(1, 2).contiguous())
    if bias is not None:
        z = z + bias.double()[:, None]
    classes = z.shape[-1]
    ok = (labels >= 0) & (labels < classes)
    c = ok.sum(-1).clamp(min=1).double()
    at = labels.long().clamp(0, classes - 1)[..., None]
    lse = torch.logsumexp(z, -1)
    loss = torch.where(ok, lse - z.gather(-1, at)[..., 0], torch.zeros_like(lse))
    dz = torch.exp(z - lse[..., None])
    dz.scatter_add_(-1, at, torch.full_like(lse, -1.0)[..., None])
    dz = torch.where(ok[..., None], dz, torch.zeros_like(dz)) / c[:, None, None]
    return loss, loss.sum(-1) / c, torch.matmul(dz, w.double()), torch.matmul(dz.transpose(1, 2).contiguous(), h.double()), dz.sum(1), dz


def rel(a, b):
    b = b.double()
    n = b.norm()
    d = (a.double() - b).norm()
    return float(d / n) if n > 0 else float(d)


def strided(t, row_pad=0, rep_pad=0, offset=0):
    """The values of t [N, rows, cols] in memory with other strides, NaN (or -77) between them."""
    n, r, c = t.shape
    row = c + row_pad
    rep = r * row + rep_pad
    fill = float("nan") if t.is_floating_point() else -77
    buf = torch.full((offset + n * rep + 64,), fill, dtype=t.dtype, device=t.device)
    v = torch.as_strided(buf, (n, r, c), (rep, row, 1), offset)
    v.copy_(t)
    return v
