"""Rotated heads, masked attention and clipped gradients in 64 bits, from their formulas, and the error bounds that the tests of the kernels hold them to.

U = 2^-24 and, for bfloat16, B = 2^-8 are half a step relative to a number of the type.  Bounds are per element, from the sizes of the terms of each sum.
"""
import math

import torch

U = 2.0 ** -24
DEV = "cuda:0"


def half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


# ---- rotation -----------------------------------------------------------------------------------
def frequencies(rotated, base=10000.0):
    return torch.tensor([base ** (-2.0 * t / rotated) for t in range(rotated // 2)], dtype=torch.float64, device=DEV)


def turn(u, pos, freq, paired, magnitude, back=False):
    """u [N, rows, heads, d] (fp64) with its first 2 len(freq) columns turned."""
    r = 0 if freq is None else 2 * freq.numel()
    if r == 0:
        return u
    a = pos.double()[..., None] * freq
    c, s = torch.cos(a)[:, :, None] * magnitude, torch.sin(a)[:, :, None] * magnitude * (-1.0 if back else 1.0)
    out = u.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if paired else (slice(0, r // 2), slice(r // 2, r))
    out[..., first] = u[..., first] * c - u[..., second] * s
    out[..., second] = u[..., first] * s + u[..., second] * c
    return out


def rotary(x, gain, d, pos, freq, paired, magnitude, eps):
    n, rows, w = x.shape
    u = x.double().view(n, rows, w // d, d)
    if gain is not None:
        u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps) * gain.double()[:, None, None]
    return turn(u, pos, freq, paired, magnitude).reshape(n, rows, w)


def rotary_backward(x, dy, gain, d, pos, freq, paired, magnitude, eps):
    n, rows, width = dy.shape
    w = turn(dy.double().view(n, rows, width // d, d), pos, freq, paired, magnitude, back=True)
    if gain is None:
        return w.reshape(n, rows, width), None, None
    u = x.double().view_as(w)
    rstd = 1.0 / torch.sqrt((u * u).mean(-1, keepdim=True) + eps)
    xh, wg = u * rstd, w * gain.double()[:, None, None]
    dx = rstd * (wg - xh * (wg * xh).mean(-1, keepdim=True))
    return dx.reshape(n, rows, width), (w * xh).sum((1, 2)), (w * xh).abs().sum((1, 2))


# ---- attention ----------------------------------------------------------------------------------
def key_ranges(n, seqs, q_len, kv_len, causal=True, window=0, positions=None, first=None, end=None, device=DEV):
    """first, end (empty: end <= first) and position of every query, [N, seqs, q_len]."""
    shape = (n, seqs, q_len)
    pos = (torch.arange(q_len, device=device) + kv_len - q_len).expand(shape) if positions is None else positions.view(shape).long()
    lo = torch.zeros(shape, dtype=torch.int64, device=device)
    hi = torch.full(shape, kv_len, dtype=torch.int64, device=device)
    if first is not None:
        lo = torch.maximum(lo, first.view(shape).long())
    if window:
        lo = torch.maximum(lo, pos - window + 1)
    if end is not None:
        hi = torch.minimum(hi, end.view(shape).long())
    if causal:
        hi = torch.minimum(hi, pos + 1)
    return lo, hi, pos


def attention(q, k, v, heads, kv_heads, seqs, dout=None, scale=None, softcap=0.0, slopes=None, **mask):
    """A dict of results (fp64, in the layout of the operator) and, under "bound_" + name, how far the kernels' may be off."""
    n, rows, width = q.shape
    d, group = width // heads, heads // kv_heads
    q_len, kv_len = rows // seqs, k.shape[1] // seqs
    scale = d ** -0.5 if scale is None else scale
    b, t = half(q.dtype), q.dtype

    def split(x, length, count):
        return x.double().view(n, seqs, length, count, d).transpose(2, 3)

    def join(x):
        return x.transpose(2, 3).reshape(n, -1, x.shape[2] * d)

    lo, hi, pos = key_ranges(n, seqs, q_len, kv_len, **mask)
    j = torch.arange(kv_len, device=q.device)
    seen = ((j >= lo[..., None]) & (j < hi[..., None]))[:, :, None]
    some = seen.any(-1, keepdim=True)
    # whatever lies in places that nothing attends takes part in nothing
    rows_seen, keys_seen = some, seen.any(-2)[..., None]
    q_, k_, v_ = split(q, q_len, heads), split(k, kv_len, kv_heads), split(v, kv_len, kv_heads)
    q_, k_, v_ = q_.masked_fill(~rows_seen, 0.0), k_.masked_fill(~keys_seen, 0.0), v_.masked_fill(~keys_seen, 0.0)
    k_, v_ = k_.repeat_interleave(group, 2), v_.repeat_interleave(group, 2)
    kt, vt = k_.transpose(-1, -2).contiguous(), v_.transpose(-1, -2).contiguous()
    z = torch.matmul(q_, kt) * scale
    # a score: products and sums in fp32, then the cap, the bias and a difference, each rounded at the size of the score
    wide = torch.matmul(q_.abs(), kt.abs()) * abs(scale)
    bend = torch.ones_like(z)
    if softcap:
        bend = 1.0 - torch.tanh(z / softcap) ** 2
        z = softcap * torch.tanh(z / softcap)
    if slopes is not None:
        bias = slopes.double().view(n, 1, heads, 1, 1) * (pos[:, :, None, :, None] - j).abs()
        z, wide = z - bias, wide + bias
    z = z.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(z, -1, keepdim=True)
    p = torch.where(some, torch.exp(z - torch.where(some, lse, torch.zeros_like(lse))), torch.zeros_like(z))
    off = U * ((d + 16) * wide.masked_fill(~seen, 0.0).amax(-1, keepdim=True) + 4.0 * softcap + 4.0 * lse.abs().masked_fill(~some, 0.0) + 16.0)
    sums = U * (kv_len + 16)                                     # of a sum over keys
    rel = 2.0 * off + sums + (b if t == torch.bfloat16 else 0.0)  # of p in a product: the score's error in it and in its row's sum
    o = torch.matmul(p, v_)
    size = torch.matmul(p, v_.abs())
    res = {"out": join(o), "bound_out": join(rel * size + b * o.abs()), "lse": lse[..., 0].transpose(1, 2).reshape(n, heads, rows),
           "bound_lse": (off + sums + 8 * U)[..., 0].transpose(1, 2).reshape(n, heads, rows)}
    if dout is None:
        return res
    do = split(dout, q_len, heads).masked_fill(~rows_seen, 0.0)
    dp, dp_size = torch.matmul(do, vt), torch.matmul(do.abs(), vt.abs())
    dot = (do * o).sum(-1, keepdim=True)
    # do . out takes out as it is stored
    off_dot = (do.abs() * (rel * size + b * o.abs())).sum(-1, keepdim=True) + U * (d + 8) * (do.abs() * size).sum(-1, keepdim=True)
    dz = p * (dp - dot) * bend
    off_bend = 8.0 * U + 2.0 * off / softcap if softcap else 0.0
    off_dz = p * (off_dot + U * (d + 8) * dp_size) + dz.abs() * (2.0 * off + 8.0 * U) + p * (dp - dot).abs() * off_bend + b * dz.abs()
    rows_sum = U * (q_len * group + 16)

    def shared(x):
        return join(x.view(n, seqs, kv_heads, group, kv_len, d).sum(3))

    def t_(x):
        return x.transpose(-1, -2).contiguous()

    dq = torch.matmul(dz, k_) * scale
    dk, dv = torch.matmul(t_(dz), q_) * scale, torch.matmul(t_(p), do)
    res["dq"], res["dk"], res["dv"] = join(dq), shared(dk), shared(dv)
    res["bound_dq"] = join(torch.matmul(off_dz + sums * dz.abs(), k_.abs()) * abs(scale)) + (b + 4 * U) * res["dq"].abs()
    res["bound_dk"] = shared(torch.matmul(t_(off_dz + rows_sum * dz.abs()), q_.abs()) * abs(scale)) + (b + 4 * U) * res["dk"].abs()
    res["bound_dv"] = shared(torch.matmul(t_(p * (2.0 * off + rows_sum + (b if t == torch.bfloat16 else 0.0))), do.abs())) + (b + 4 * U) * res["dv"].abs()
    return res


def check(got, want, bound, name):
    """Element by element, and no NaN or infinity where there is none in `want`."""
    g = got.double()
    same = (g == want) | ((g != g) & (want != want))
    bad = ~same & ~((g - want).abs() <= bound * 1.01 + 1e-40)
    if bool(bad.any()):
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, the first at {at}: {float(g[at])} for {float(want[at])}, bound {float(bound[at])}")
