"""Performance cases of the language-model operators: the calls that a program makes which trains N replicas of a language
model with 8-bit linear layers, and which then answers with them.

A case is one pass through the public binding on buffers laid out as such a program keeps them, [replica][row][column]:
  kind "norm"    root-mean-square norm of a residual sum with its output in 8 bits, the 8-bit copy read back, and the backward pass
  kind "serve"   the norm and the 8-bit linear layer behind it, for the few rows of a decoding step
  kind "linear"  the 8-bit linear layer; with "back", its gradients from the 8-bit copies of input and weight too
  kind "loss"    the output layer with its cross-entropy, in pieces of the vocabulary, with all its gradients
Where `own` is false, run() evaluates the same in elementary tensor operations in 32 bits; exact() in 64 bits.

Rows in 8 bits: codes -127 .. 127 and one scale a row, the smallest power of two (2^-126 at least) that takes the row's largest entry
to 127 or less; a code is the entry over the scale, rounded to the nearest whole number, halves to even.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the norm in front of a block of the 6-layer, 512-wide transformer: 16 sequences of 256 tokens, 8 replicas
        dict(name="norm_6l", kind="norm", n=8, rows=4096, width=512, dtype="bf16"),
        # the same of the 12-layer, 1024-wide one: 16 sequences of 512
        dict(name="norm_12l", kind="norm", n=8, rows=8192, width=1024, dtype="bf16"),
        # a full-precision study of odd width and length
        dict(name="norm_f32_odd", kind="norm", n=3, rows=777, width=1001, dtype="f32"),
        # one token a replica through norm and first MLP layer: latency
        dict(name="serve_one_token", kind="serve", n=8, rows=1, d_in=512, d_out=2048),
        # 16 sequences a replica decoded together: the weights' stream
        dict(name="serve_16_tokens", kind="serve", n=8, rows=16, d_in=1024, d_out=4096),
        # first MLP layer of the 6-layer transformer, forward (evaluation of the replicas)
        dict(name="linear_6l", kind="linear", n=8, rows=4096, d_in=512, d_out=2048, dtype="bf16", back=False),
        # first MLP layer of the 12-layer transformer, with its gradients
        dict(name="linear_12l_train", kind="linear", n=8, rows=8192, d_in=1024, d_out=4096, dtype="bf16", back=True),
        # a ragged batch through a layer of ragged widths, results in full precision
        dict(name="linear_ragged_train", kind="linear", n=3, rows=515, d_in=776, d_out=1501, dtype="f32", back=True),
        # the smallest transformer study's head: launches and latency
        dict(name="loss_small", kind="loss", n=4, rows=128, width=64, classes=512, dtype="f32"),
        # a vocabulary of odd size, weight gradients in full precision
        dict(name="loss_ragged", kind="loss", n=2, rows=1000, width=776, classes=5003, dtype="f32"),
        # head of the 6-layer transformer
        dict(name="loss_6l", kind="loss", n=8, rows=4096, width=512, classes=32000, dtype="bf16"),
        # head of the 12-layer transformer, weight gradients in full precision as the optimizer takes them
        dict(name="loss_12l", kind="loss", n=4, rows=8192, width=1024, classes=32000, dtype="f32"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v - 1 if v == 3072 else v


def _size(rng, lo, hi):
    """A width: as often as not a multiple of 64 as layers have, else any number."""
    v = _log(rng, lo, hi)
    v = max(lo, (v + 32) // 64 * 64) if rng.random() < 0.5 else v
    return v - 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(["norm", "serve", "linear", "linear", "loss", "loss"])
    n = rng.choice([1, 2, 3, 4, 5, 8])
    if kind == "norm":
        width = _size(rng, 64, 8192)
        return dict(kind="norm", n=n, rows=_log(rng, 1, max(1, 32_000_000 // (n * width))), width=width, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "serve":
        return dict(kind="serve", n=n, rows=_log(rng, 1, 32), d_in=_size(rng, 64, 8192), d_out=_size(rng, 64, 4096))
    if kind == "linear":
        d_in, d_out = _size(rng, 64, 8192), _size(rng, 64, 4096)
        rows = _log(rng, 1, max(1, min(16384, 250_000_000_000 // (2 * n * d_in * d_out), 60_000_000 // (n * max(d_in, d_out)))))
        return dict(kind="linear", n=n, rows=rows, d_in=d_in, d_out=d_out, dtype=rng.choice(["bf16", "f32"]), back=rng.random() < 0.6)
    width, classes = _size(rng, 64, 2048), _size(rng, 100, 64000)
    rows = _log(rng, 1, max(1, min(8192, 400_000_000 // (n * classes), 250_000_000_000 // (n * classes * width))))
    return dict(kind="loss", n=n, rows=rows, width=width, classes=classes, dtype=rng.choice(["bf16", "f32"]))


def _rows8(v):
    """Codes and scales of the rows of v, in v's precision."""
    m, k = torch.frexp(v.abs().amax(-1, keepdim=True))
    e = (k - 7 + (m > 127.0 / 128.0).to(k.dtype)).clamp(min=-126)
    e = torch.where(m == 0, torch.full_like(e, -126), e)
    s = torch.ldexp(torch.ones_like(m), e)
    return torch.round(v / s), s


def _padded(codes):
    """Codes as 8-bit rows that start 16 bytes apart, zeros behind the last column."""
    w = codes.shape[-1]
    out = torch.zeros(*codes.shape[:-1], (w + 15) // 16 * 16, dtype=torch.int8, device=codes.device)
    out[..., :w] = codes.to(torch.int8)
    return out[..., :w]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    f32 = dict(dtype=torch.float32, device=DEV)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)

    n = case["n"]
    s = dict(kind=case["kind"], case=case)
    if case["kind"] in ("norm", "serve"):
        rows, width = case["rows"], case["width"] if case["kind"] == "norm" else case["d_in"]
        dt = TYPES[case.get("dtype", "bf16")]
        # a residual stream whose rows differ in size and have a few large columns, and what a block adds to it
        big = 1.0 + 7.0 * (torch.rand(width, generator=g, device=DEV) < 0.02)
        s["x"] = (normal(n, rows, width) * big * torch.exp(normal(n, rows, 1, std=0.5))).to(dt)
        s["resid"] = normal(n, rows, width, std=0.5, dtype=dt)
        s["gain"] = 1.0 + normal(n, width, std=0.1)
        s["total"] = torch.empty_like(s["x"])
        s["codes"] = _padded(torch.zeros(n, rows, width, **f32))
        s["scale"] = torch.empty(n, rows, **f32)
        s["rstd"] = torch.empty(n, rows, **f32)
    if case["kind"] == "norm":
        s["dy"], s["dtotal"] = normal(n, rows, width, std=1e-3, dtype=dt), normal(n, rows, width, std=1e-3, dtype=dt)
        s["values"] = torch.empty(n, rows, width, dtype=torch.bfloat16, device=DEV)
        s["dx"] = torch.empty_like(s["x"])
        s["dgain"] = torch.empty(n, width, **f32)
    if case["kind"] in ("serve", "linear"):
        rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
        dt = TYPES[case.get("dtype", "bf16")]
        w, ws = _rows8(normal(n, d_out, d_in, std=d_in ** -0.5))
        s["w_codes"], s["w_scale"] = _padded(w), ws[..., 0].contiguous()
        s["bias"] = normal(n, d_out, std=0.1)
        s["y"] = torch.empty(n, rows, d_out, dtype=dt, device=DEV)
    if case["kind"] == "linear":
        x, xs = _rows8(normal(n, rows, d_in) * torch.exp(normal(n, rows, 1, std=0.5)))
        s["codes"], s["scale"] = _padded(x), xs[..., 0].contiguous()
        if case["back"]:
            s["dy"] = normal(n, rows, d_out, std=1e-3, dtype=torch.bfloat16)
            s["dx"] = torch.empty(n, rows, d_in, dtype=torch.bfloat16, device=DEV)
            s["dw"], s["db"] = torch.empty(n, d_out, d_in, **f32), torch.empty(n, d_out, **f32)
    if case["kind"] == "loss":
        rows, width, classes, dt = case["rows"], case["width"], case["classes"], TYPES[case["dtype"]]
        s["h"] = normal(n, rows, width, dtype=torch.bfloat16)
        s["w"] = normal(n, classes, width, std=2.0 * width ** -0.5, dtype=torch.bfloat16)
        s["bias"] = normal(n, classes, std=0.1)
        # next tokens by Zipf's law; one in sixteen is padding and counts for nothing (the first row never is)
        p = 1.0 / torch.arange(1, classes + 1, dtype=torch.float64, device=DEV) ** 1.1
        ids = torch.searchsorted(torch.cumsum(p, 0) / p.sum(), torch.rand(n, rows, generator=g, device=DEV, dtype=torch.float64))
        pad = torch.rand(n, rows, generator=g, device=DEV) < 1.0 / 16.0
        pad[:, 0] = False
        s["labels"] = torch.where(pad, torch.full_like(ids, -1), ids.clamp(max=classes - 1)).to(torch.int32)
        s["row_loss"], s["mean"] = torch.empty(n, rows, **f32), torch.empty(n, **f32)
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty(n, classes, width, dtype=dt, device=DEV)
        s["db"] = torch.empty(n, classes, **f32)
    return s


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    import paper_2604_24708_amd as H

    def work(size):
        # kept with the state, as a training program keeps it between its steps
        if "work" not in s:
            s["work"] = torch.empty(max(size(), 16), dtype=torch.uint8, device=DEV)
        return s["work"]

    stream = torch.cuda.current_stream().cuda_stream
    kind, c = s["kind"], s["case"]
    if kind in ("norm", "serve"):
        H.hdet_rmsnorm(s["x"], s["gain"], resid=s["resid"], total=s["total"], codes=s["codes"], scale=s["scale"],
                       rstd=s["rstd"] if kind == "norm" else None, eps=EPS, stream=stream)
    if kind == "norm":
        H.hdet_restore_rows(s["codes"], s["scale"], s["values"], stream=stream)
        H.hdet_rmsnorm_backward(s["total"], s["gain"], s["rstd"], s["dy"], s["dx"], dtotal=s["dtotal"], dgain=s["dgain"],
                                workspace=work(lambda: H.hdet_rmsnorm_backward_workspace(c["n"], c["rows"], c["width"])), stream=stream)
        return {"total": s["total"], "values": s["values"], "rstd": s["rstd"], "dx": s["dx"], "dgain": s["dgain"]}
    if kind in ("serve", "linear"):
        H.hdet_quantised_linear(s["codes"], s["scale"], s["w_codes"], s["w_scale"], s["y"], bias=s["bias"], stream=stream)
    if kind == "serve":
        return {"total": s["total"], "y": s["y"]}
    if kind == "linear":
        if not c["back"]:
            return {"y": s["y"]}
        H.hdet_quantised_linear_backward(
            s["dy"], s["codes"], s["scale"], s["w_codes"], s["w_scale"], dx=s["dx"], dw=s["dw"], db=s["db"],
            workspace=work(lambda: H.hdet_quantised_linear_backward_workspace(c["n"], c["rows"], c["d_in"], c["d_out"])), stream=stream)
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    H.hdet_vocab_loss(s["h"], s["w"], s["labels"], s["row_loss"], s["mean"], dh=s["dh"], dw=s["dw"], bias=s["bias"], db=s["db"],
                      workspace=work(lambda: H.hdet_vocab_loss_workspace(c["n"], c["rows"], c["width"], c["classes"], dw=s["dw"].dtype)), stream=stream)
    return {"loss": s["row_loss"], "mean": s["mean"], "dh": s["dh"], "dw": s["dw"], "db": s["db"]}


def _plain_norm(s):
    u = s["x"].float() + s["resid"].float()
    rstd = torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS)
    q, scale = _rows8(u * rstd * s["gain"][:, None])
    return u, rstd, q, scale


def _plain_linear(s, x):
    w = s["w_codes"].float() * s["w_scale"][..., None]
    return w, torch.matmul(x, w.transpose(1, 2)) + s["bias"][:, None]


def _plain(s):
    kind = s["kind"]
    if kind == "norm":
        dt = s["x"].dtype
        u, rstd, q, scale = _plain_norm(s)
        # the backward pass has the sum as it is stored
        xhat = u.to(dt).float() * rstd
        dy = s["dy"].float()
        dn = dy * s["gain"][:, None]
        dx = rstd * (dn - xhat * (dn * xhat).mean(-1, keepdim=True)) + s["dtotal"].float()
        return {"total": u.to(dt), "values": (q * scale).to(torch.bfloat16), "rstd": rstd[..., 0], "dx": dx.to(dt), "dgain": (dy * xhat).sum(1)}
    if kind == "serve":
        u, _, q, scale = _plain_norm(s)
        _, y = _plain_linear(s, q * scale)
        return {"total": u.to(s["x"].dtype), "y": y.to(s["y"].dtype)}
    if kind == "linear":
        x = s["codes"].float() * s["scale"][..., None]
        w, y = _plain_linear(s, x)
        if not s["case"]["back"]:
            return {"y": y.to(s["y"].dtype)}
        dy = s["dy"].float()
        return {"y": y.to(s["y"].dtype), "dx": torch.matmul(dy, w).to(torch.bfloat16), "dw": torch.matmul(dy.transpose(1, 2), x), "db": dy.sum(1)}
    h, w, lab = s["h"].float(), s["w"].float(), s["labels"].long()
    z = torch.matmul(h, w.transpose(1, 2)) + s["bias"][:, None]
    top = z.amax(-1, keepdim=True)
    z -= top
    counts = (lab >= 0) & (lab < z.shape[-1])
    at = lab.clamp(0, z.shape[-1] - 1)[..., None]
    zy = z.gather(-1, at)
    p = z.exp_()
    total = p.sum(-1, keepdim=True)
    row = torch.where(counts, (total.log() - zy)[..., 0], torch.zeros_like(total[..., 0]))
    number = counts.sum(-1, keepdim=True).clamp(min=1).float()
    p *= (counts / number)[..., None] / total
    p.scatter_add_(-1, at, -(counts / number)[..., None])
    return {"loss": row, "mean": row.sum(-1) / number[..., 0], "dh": torch.matmul(p, w).to(s["h"].dtype),
            "dw": torch.matmul(p.transpose(1, 2), h).to(s["dw"].dtype), "db": p.sum(1)}


def work(case):
    n, k = case["n"], case["kind"]
    if k == "norm":
        e, b = n * case["rows"] * case["width"], 2 if case["dtype"] == "bf16" else 4
        # in: the two summands and the two gradients; out: the sum, its gradient, the 8-bit copy and the values it stands for
        return {"bytes": e * (6 * b + 1 + 2) + n * (case["rows"] * 8 + case["width"] * 8), "flops": 24 * e}
    if k == "loss":
        rows, d, v = case["rows"], case["width"], case["classes"]
        b = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * (rows * d * 4 + v * d * (2 + b) + v * 8 + rows * 8), "flops": 6 * n * rows * d * v}
    rows, i, o = case["rows"], case["d_in"], case["d_out"]
    y = 2 if case.get("dtype", "bf16") == "bf16" else 4
    r = {"bytes": n * (i * o + o * 8 + rows * o * y), "flops": 2 * n * rows * i * o}
    if k == "serve":
        r["bytes"] += n * (rows * i * 6 + i * 4)
        return r
    r["bytes"] += n * rows * (i + 4)
    if case["back"]:
        r["bytes"] += n * (rows * o * 2 + rows * i * 2 + i * o * 4 + o * 4)
        r["flops"] *= 3
    return r


def _exact_norm(s):
    u = s["x"].double() + s["resid"].double()
    rstd = 1.0 / torch.sqrt(u.square().sum(-1) / u.shape[-1] + EPS)
    y = u * rstd[:, :, None] * s["gain"].double()[:, None, :]
    top = y.abs().max(-1).values
    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 127.0)).clamp(min=-126.0)
    scale = torch.pow(torch.full_like(e, 2.0), e)[:, :, None]
    return u, rstd, torch.round(y / scale) * scale


def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "norm":
        u, rstd, v = _exact_norm(s)
        w = s["x"].shape[-1]
        stored = u.to(s["x"].dtype).double()
        dy, t = s["dy"].double(), s["gain"].double()[:, None, :]
        dot = (dy * t * stored).sum(-1)
        dx = dy * t * rstd[:, :, None] - stored * (dot * rstd ** 3 / w)[:, :, None] + s["dtotal"].double()
        return {"total": u, "values": v, "rstd": rstd, "dx": dx, "dgain": torch.einsum("nrd,nr->nd", dy * stored, rstd)}
    if k in ("serve", "linear"):
        total = None
        if k == "serve":
            total, _, x = _exact_norm(s)
        else:
            x = s["codes"].double() * s["scale"].double().unsqueeze(-1)
        out = {"y": [], "dx": [], "dw": [], "db": []}
        for r in range(case["n"]):
            w = s["w_codes"][r].double() * s["w_scale"][r].double().unsqueeze(-1)
            out["y"].append(x[r] @ w.t().contiguous() + s["bias"][r].double())
            if case.get("back"):
                dy = s["dy"][r].double()
                out["dx"].append(dy @ w)
                out["dw"].append(dy.t().contiguous() @ x[r])
                out["db"].append(dy.sum(0))
        got = {key: torch.stack(v) for key, v in out.items() if v}
        if total is not None:
            got["total"] = total
        return got
    rows, classes = case["rows"], case["classes"]
    out = {"loss": [], "mean": [], "dh": [], "dw": [], "db": []}
    for r in range(case["n"]):
        h, w, lab = s["h"][r].double(), s["w"][r].double(), s["labels"][r].long()
        ok = torch.nonzero((lab >= 0) & (lab < classes))[:, 0]
        h2, lab2 = h[ok], lab[ok]
        z = h2 @ w.t().contiguous() + s["bias"][r].double()
        lse = torch.logsumexp(z, 1)
        one = lse - z[torch.arange(len(ok), device=DEV), lab2]
        loss = torch.zeros(rows, dtype=torch.float64, device=DEV)
        loss[ok] = one
        p = torch.exp(z - lse[:, None])
        del z
        p[torch.arange(len(ok), device=DEV), lab2] -= 1.0
        p /= len(ok)
        dh = torch.zeros(rows, case["width"], dtype=torch.float64, device=DEV)
        dh[ok] = p @ w
        for key, v in zip(("loss", "mean", "dh", "dw", "db"), (loss, one.mean(), dh, p.t() @ h2, p.sum(0))):
            out[key].append(v)
        del p
    return {key: torch.stack(v) for key, v in out.items()}
