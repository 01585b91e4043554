"""Performance cases of the operators between a language model's linear layers and behind its backward pass: rotated heads, attention
under the masks of packed, prefixed and cached sequences, and the clipped gradient that the update takes.

A case is one pass through the public binding on buffers laid out as a program keeps them that trains N replicas (and answers with them),
[replica][token][head and column]:
  kind "rotate"  norm of every head of the queries and keys with the rotation by position; with "back", the gradients too
  kind "attend"  attention; with "back", the gradients too
  kind "clip"    the norm of each replica's gradient over all tensors of a model, and the clipped gradient in the plane of the update
Where `own` is false, run() evaluates the same in elementary tensor operations in 32 bits (angles and norms in 64); exact() in 64 bits.

Which keys a query attends is a range of its sequence, first .. end - 1, as a data loader hands it out with the tokens ("mask"):
  "causal"   up to itself
  "packed"   up to itself in its own document; what is left of a sequence behind its last document attends nothing
  "prefix"   all of the sequence's first part, and up to itself; the sequences' ends are padding
  "cache"    the tokens that the sequence has so far in a cache with room for more
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # decoding step of the 12-layer transformer: one token of 16 sequences a replica, far into a long context
        dict(name="rotate_one_token", kind="rotate", n=8, seqs=16, q_len=1, heads=16, kv_heads=4, d=64, rotated=64, paired=False, norm=True, far=100000, stretch=8.0,
             dtype="bf16", back=False),
        # the 6-layer transformer's step: 16 sequences of 256 tokens
        dict(name="rotate_6l_train", kind="rotate", n=8, seqs=16, q_len=256, heads=8, kv_heads=8, d=64, rotated=64, paired=False, norm=True, far=0, stretch=1.0,
             dtype="bf16", back=True),
        # the 12-layer one's with shared key heads, pairs next to each other, half of the head
        dict(name="rotate_12l_train", kind="rotate", n=8, seqs=16, q_len=512, heads=16, kv_heads=4, d=64, rotated=32, paired=True, norm=True, far=0, stretch=1.0,
             dtype="bf16", back=True),
        # a full-precision study of odd lengths and heads
        dict(name="rotate_f32_odd", kind="rotate", n=3, seqs=1, q_len=777, heads=5, kv_heads=1, d=50, rotated=18, paired=False, norm=True, far=5000, stretch=4.0,
             dtype="f32", back=True),
        # the smallest transformer study, in fp32: launches and latency
        dict(name="attend_small_train", kind="attend", n=4, seqs=4, q_len=32, kv_len=32, heads=4, kv_heads=4, d=16, mask="causal", window=0, cap=0.0, slopes=False,
             dtype="f32", back=True),
        # attention of the 6-layer transformer
        dict(name="attend_6l_train", kind="attend", n=8, seqs=16, q_len=256, kv_len=256, heads=8, kv_heads=8, d=64, mask="causal", window=0, cap=0.0, slopes=False,
             dtype="bf16", back=True),
        # the 12-layer one's on packed documents, shared key heads, capped scores
        dict(name="attend_12l_packed_train", kind="attend", n=8, seqs=16, q_len=512, kv_len=512, heads=16, kv_heads=4, d=64, mask="packed", window=0, cap=30.0,
             slopes=False, dtype="bf16", back=True),
        # a ragged batch of prompts with their answers, heads of no whole tile, scores that fall with the distance
        dict(name="attend_ragged_train", kind="attend", n=3, seqs=2, q_len=333, kv_len=333, heads=6, kv_heads=2, d=72, mask="prefix", window=0, cap=0.0, slopes=True,
             dtype="bf16", back=True),
        # evaluation on a long sequence
        dict(name="attend_long", kind="attend", n=2, seqs=1, q_len=8192, kv_len=8192, heads=8, kv_heads=2, d=128, mask="causal", window=0, cap=0.0, slopes=False,
             dtype="bf16", back=False),
        # decoding: one token of 16 sequences a replica over their caches
        dict(name="attend_one_token", kind="attend", n=8, seqs=16, q_len=1, kv_len=4096, heads=16, kv_heads=4, d=64, mask="cache", window=0, cap=0.0, slopes=False,
             dtype="bf16", back=False),
        # the smallest transformer study's gradient: many short tensors
        dict(name="clip_small", kind="clip", n=4, blocks=2, width=64, ff=256, vocab=512, shared=False, wide="f32"),
        # the 12-layer transformer's, the embeddings' gradients in bfloat16
        dict(name="clip_12l", kind="clip", n=4, blocks=12, width=1024, ff=4096, vocab=32000, shared=False, wide="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8])
    return kv * rng.choice([1, 1, 2, 4]), kv


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "attend", "attend", "attend", "decode", "clip"])
    n = rng.choice([1, 2, 3, 4, 5, 8])
    if kind == "clip":
        width = _log(rng, 32, 1024)
        width = width // 16 * 16 if rng.random() < 0.5 else width
        vocab, ff = _log(rng, 100, 32000), _log(rng, 2 * width, 4 * width)
        most = 800_000_000 // n - 2 * vocab * width
        blocks = max(1, min(rng.randint(1, 12), most // (4 * width * width + 2 * width * ff)))
        return dict(kind="clip", n=n, blocks=blocks, width=width, ff=ff, vocab=vocab, shared=rng.random() < 0.4, wide=rng.choice(["f32", "bf16"]))
    heads, kv_heads = _heads(rng)
    d = rng.choice([64, 64, 128, 32, 16, 80, 96, rng.randint(4, 128)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rotate":
        back = rng.random() < 0.6
        rows = _log(rng, 1, max(1, min(131072, 80_000_000 // (n * (heads + kv_heads) * d))))
        seqs = rng.choice([1, 2, 16])
        q_len = max(1, rows // seqs)
        return dict(kind="rotate", n=n, seqs=seqs, q_len=q_len, heads=heads, kv_heads=kv_heads, d=d, rotated=rng.choice([d // 2 * 2, d // 4 * 2, d // 2 * 2]),
                    paired=rng.random() < 0.4, norm=rng.random() < 0.8, far=rng.choice([0, 0, _log(rng, 1000, 1000000)]), stretch=rng.choice([1.0, 4.0, 32.0]), dtype=dtype,
                    back=back)
    if kind == "decode":
        seqs = rng.choice([1, 2, 5, 16])
        kv_len = _log(rng, 64, max(64, min(65536, 120_000_000 // (n * seqs * kv_heads * d))))
        return dict(kind="attend", n=n, seqs=seqs, q_len=rng.choice([1, 1, 1, 2, 5]), kv_len=kv_len, heads=heads, kv_heads=kv_heads, d=d, mask="cache",
                    window=rng.choice([0, 0, 0, max(1, kv_len // 3)]), cap=rng.choice([0.0, 0.0, 30.0]), slopes=rng.random() < 0.2, dtype=dtype, back=False)
    back = rng.random() < 0.7
    f32 = dtype == "f32"
    pairs = (150_000_000 if f32 else 500_000_000) // n // heads * min(64, d) // d
    q_len = _log(rng, 2, max(2, min(8192, int(pairs ** 0.5))))
    if rng.random() < 0.4:
        q_len = max(2, q_len // 64 * 64)
    seqs = max(1, min(rng.choice([1, 2, 5, 16]), pairs // (q_len * q_len)))
    return dict(kind="attend", n=n, seqs=seqs, q_len=q_len, kv_len=q_len, heads=heads, kv_heads=kv_heads, d=d, mask=rng.choice(["causal", "packed", "packed", "prefix"]),
                window=rng.choice([0, 0, 0, max(2, q_len // 4)]), cap=rng.choice([0.0, 0.0, 30.0]), slopes=rng.random() < 0.3, dtype=dtype, back=back)


# ---- inputs -----------------------------------------------------------------------------------------
def _shapes(case):
    """Tensors of a transformer's parameters: biases and gains are [columns], the others [rows][columns]."""
    w, ff, v = case["width"], case["ff"], case["vocab"]
    out = [(v, w)]
    for _ in range(case["blocks"]):
        out += [(w,), (w, w), (w, w), (w, w), (w, w), (w,), (ff, w), (ff,), (w, ff), (w,)]
    return out + [(w,), (v, w), (v,)]


def _key_ranges(case, seed):
    """first, end, position of every query, [replica][sequence][query] (CPU)."""
    rng = random.Random(seed)
    n, b, ql, kl = case["n"], case["seqs"], case["q_len"], case["kv_len"]
    i = torch.arange(ql)
    first, end, pos = [], [], []
    for _ in range(n * b):
        p = i + kl - ql
        f, e = torch.zeros(ql, dtype=torch.int64), p + 1
        if case["mask"] == "packed":
            e = torch.zeros(ql, dtype=torch.int64)
            at, last = 0, ql - rng.randint(0, ql // 8)
            while at < last:
                stop = min(last, at + 1 + int(rng.expovariate(3.0 / ql)))
                f[at:stop] = at
                e[at:stop] = i[at:stop] + 1
                at = stop
        elif case["mask"] == "prefix":
            have = ql - rng.randint(0, ql // 4)
            e = torch.clamp(i + 1, min=rng.randint(0, have // 2))
            e[have:] = 0
        elif case["mask"] == "cache":
            p = i + rng.randint(kl // 4, kl - ql) if kl >= 2 * ql else i + kl - ql
            e = p + 1
        if case["window"]:
            f = torch.maximum(f, p - case["window"] + 1)
        first.append(f)
        end.append(e)
        pos.append(p)
    return [torch.stack(x).view(n, b, ql) for x in (first, end, pos)]


def _frequencies(case):
    """Radians a position for each pair; with "stretch", pairs that turn less than once over 2048 positions go that much slower, those that turn more than 32 times as
    they were, the others in between."""
    r = case["rotated"]
    if r == 0:
        return torch.zeros(0, dtype=torch.float64, device=DEV)
    f = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
    keep = ((2048.0 * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / case["stretch"])


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)

    n, kind = case["n"], case["kind"]
    s = dict(kind=kind, case=case)
    if kind == "clip":
        s["grads"], at, places = [], 0, []
        shapes = _shapes(case)
        for shape in shapes:
            places.append(at)
            at += -(-math.prod(shape) // 4) * 4
        stride = -(-at // 64) * 64
        # the plane of the update: tensors at multiples of four elements, zeros between them
        s["plane"] = torch.zeros(n, stride, device=DEV)
        s["outs"] = [s["plane"][:, p:p + math.prod(shape)].view(n, *shape) for p, shape in zip(places, shapes)]
        size = (torch.arange(n, device=DEV, dtype=torch.float32) + 1.0) * 1e-3
        for k, shape in enumerate(shapes):
            wide = k == 0 or k == len(shapes) - 2
            x = normal(n, *shape).mul_(size.view(n, *([1] * len(shape))))
            s["grads"].append(x.to(TYPES[case["wide"]] if wide else torch.float32))
        # about half of the replicas are above it
        s["max_norm"] = float(1e-3 * (0.5 * n + 0.75) * math.sqrt(sum(math.prod(x) for x in shapes)))
        if case["shared"]:
            s["max_norm"] *= 0.5 / math.sqrt(n)
        s["norm"] = torch.empty(n, device=DEV)
        return s
    dt = TYPES[case["dtype"]]
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    rows = case["seqs"] * case["q_len"]
    if kind == "rotate":
        # queries and keys as one product of the layer below gives them, some columns larger than the others
        big = 1.0 + 3.0 * (torch.rand((h + hk) * d, generator=g, device=DEV) < 0.05)
        s["qk"] = (normal(n, rows, (h + hk) * d) * big).to(dt)
        s["out"] = torch.empty_like(s["qk"])
        s["q_gain"], s["k_gain"] = (1.0 + normal(n, d, std=0.1) for _ in range(2))
        s["freq"] = _frequencies(case)
        start = torch.randint(0, case["far"] + 1, (n, case["seqs"], 1), generator=g, device=DEV)
        s["pos"] = (start + torch.arange(case["q_len"], device=DEV)).view(n, rows).to(torch.int32)
        if case["back"]:
            s["dout"] = normal(n, rows, (h + hk) * d, std=1e-3, dtype=dt)
            s["dqk"] = torch.empty_like(s["qk"])
            s["dq_gain"], s["dk_gain"] = (torch.empty(n, d, device=DEV) for _ in range(2))
        return s
    keys = case["seqs"] * case["kv_len"]
    s["q"], s["k"], s["v"] = normal(n, rows, h * d, dtype=dt), normal(n, keys, hk * d, dtype=dt), normal(n, keys, hk * d, dtype=dt)
    s["first"], s["end"], s["pos"] = (x.reshape(n, rows).to(torch.int32).to(DEV) for x in _key_ranges(case, seed))
    s["slopes"] = (2.0 ** (-8.0 * (torch.arange(h, device=DEV, dtype=torch.float32) + 1.0) / h)).expand(n, h).contiguous() if case["slopes"] else None
    s["out"] = torch.empty_like(s["q"])
    if case["back"]:
        s["lse"] = torch.empty(n, h, rows, device=DEV)
        s["dout"] = normal(n, rows, h * d, std=1e-3, dtype=dt)
        s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
    return s


def run(s):
    return (_own if own else _plain)(s)


# ---- the framework's calls --------------------------------------------------------------------------
def _own(s):
    import paper_2604_24708_amd as H

    def work(size):
        # kept with the state, as a program keeps it between its steps
        if "work" not in s:
            s["work"] = torch.empty(max(size(), 16), dtype=torch.uint8, device=DEV)
        return s["work"]

    stream = torch.cuda.current_stream().cuda_stream
    kind, c = s["kind"], s["case"]
    n = c["n"]
    if kind == "clip":
        # where the gradients lie and where they go stays the same from step to step
        if "list" not in s:
            s["list"] = H.hdet_gradient_list(s["grads"], s["outs"])
        H.hdet_clip_gradients(s["list"], s["norm"], s["max_norm"], shared=c["shared"],
                              workspace=work(lambda: H.hdet_clip_gradients_workspace(n, len(s["grads"]))), stream=stream)
        return {"norm": s["norm"], "plane": s["plane"]}
    h, hk, d, rows = c["heads"], c["kv_heads"], c["d"], c["seqs"] * c["q_len"]
    if kind == "rotate":
        at = h * d
        gains = dict(q_gain=s["q_gain"], k_gain=s["k_gain"]) if c["norm"] else {}
        how = dict(freq=s["freq"], positions=s["pos"], paired=c["paired"], eps=EPS, stream=stream, **gains)
        H.hdet_head_rotary(s["qk"][..., :at], s["out"][..., :at], d, k=s["qk"][..., at:], k_out=s["out"][..., at:], **how)
        if not c["back"]:
            return {"out": s["out"]}
        if c["norm"]:
            how.update(dq_gain=s["dq_gain"], dk_gain=s["dk_gain"], workspace=work(lambda: H.hdet_head_rotary_backward_workspace(n, rows, d, h, hk)))
        H.hdet_head_rotary_backward(s["qk"][..., :at], s["dout"][..., :at], s["dqk"][..., :at], d, k=s["qk"][..., at:], dk_out=s["dout"][..., at:],
                                    dk=s["dqk"][..., at:], **how)
        out = {"out": s["out"], "dqk": s["dqk"]}
        if c["norm"]:
            out.update(dq_gain=s["dq_gain"], dk_gain=s["dk_gain"])
        return out
    how = dict(causal=False, softcap=c["cap"], slopes=s["slopes"], positions=s["pos"], first=s["first"], end=s["end"], stream=stream)
    if c["mask"] == "causal":
        how.update(causal=True, window=c["window"], positions=None, first=None, end=None)
    sizes = (n, c["seqs"], c["q_len"], c["kv_len"], h, hk, d)
    if not c["back"]:
        H.hdet_attention(s["q"], s["k"], s["v"], s["out"], h, hk, c["seqs"], workspace=work(lambda: H.hdet_attention_workspace(*sizes)), **how)
        return {"out": s["out"]}
    size = lambda: max(H.hdet_attention_workspace(*sizes), H.hdet_attention_backward_workspace(*sizes))  # noqa: E731
    H.hdet_attention(s["q"], s["k"], s["v"], s["out"], h, hk, c["seqs"], lse=s["lse"], workspace=work(size), **how)
    H.hdet_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], h, hk, c["seqs"], workspace=work(size), **how)
    return {"out": s["out"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


# ---- elementary tensor operations, in 32 bits -------------------------------------------------------
def _plain_pairs(x, r, paired):
    return (x[..., 0:r:2], x[..., 1:r:2]) if paired else (x[..., :r // 2], x[..., r // 2:r])


def _plain_turn(x, cos, sin, paired):
    r = 2 * cos.shape[-1]
    a, b = _plain_pairs(x, r, paired)
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((a, b), -1).flatten(-2) if paired else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_rotate(s):
    c = s["case"]
    n, h, d, rows = c["n"], c["heads"], c["d"], c["seqs"] * c["q_len"]
    x = s["qk"].float().view(n, rows, -1, d)
    angle = s["pos"].double()[..., None] * s["freq"]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    gain = torch.cat((s["q_gain"][:, None].expand(n, h, d), s["k_gain"][:, None].expand(n, c["kv_heads"], d)), 1)[:, None]
    xh = x
    if c["norm"]:
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xh = x * rstd
    y = _plain_turn(xh * gain if c["norm"] else x, cos, sin, c["paired"])
    out = {"out": y.reshape(n, rows, -1).to(s["qk"].dtype)}
    if c["back"]:
        t = _plain_turn(s["dout"].float().view_as(x), cos, -sin, c["paired"])
        dx = t
        if c["norm"]:
            tg = t * gain
            dx = rstd * (tg - xh * (tg * xh).mean(-1, keepdim=True))
            dg = t * xh
            out.update(dq_gain=dg[:, :, :h].sum((1, 2)), dk_gain=dg[:, :, h:].sum((1, 2)))
        out["dqk"] = dx.reshape(n, rows, -1).to(s["qk"].dtype)
    return out


def _plain_attend(s):
    c = s["case"]
    n, b, ql, kl, h, hk, d = (c[k] for k in ("n", "seqs", "q_len", "kv_len", "heads", "kv_heads", "d"))
    dt = s["q"].dtype

    def split(x, length, count):
        return x.float().view(n, b, length, count, d).transpose(2, 3).contiguous()

    def join(x):
        return x.transpose(2, 3).reshape(n, -1, x.shape[2] * d).to(dt)

    q, k, v = split(s["q"], ql, h), split(s["k"], kl, hk), split(s["v"], kl, hk)
    k, v = k.repeat_interleave(h // hk, 2), v.repeat_interleave(h // hk, 2)
    scale = d ** -0.5
    z = torch.matmul(q, k.transpose(-1, -2)) * scale
    if c["cap"]:
        tanh = torch.tanh(z / c["cap"])
        z = c["cap"] * tanh
    j = torch.arange(kl, device=DEV)
    first, end, pos = (s[x].view(n, b, 1, ql, 1) for x in ("first", "end", "pos"))
    if c["slopes"]:
        z = z - s["slopes"].view(n, 1, h, 1, 1) * (pos - j).abs()
    seen = (j >= first) & (j < end)
    some = seen.any(-1, keepdim=True)
    z = torch.where(seen, z, torch.full_like(z, float("-inf")))
    top = torch.where(some, z.amax(-1, keepdim=True), torch.zeros_like(z[..., :1]))
    p = torch.exp(z - top)
    p = p / torch.where(some, p.sum(-1, keepdim=True), torch.ones_like(top))
    del z
    o = torch.matmul(p, v)
    out = {"out": join(o)}
    if c["back"]:
        do = split(s["dout"], ql, h)
        ds = p * (torch.matmul(do, v.transpose(-1, -2)) - (do * o).sum(-1, keepdim=True))
        if c["cap"]:
            ds = ds * (1.0 - tanh * tanh)

        def shared(x):
            return join(x.view(n, b, hk, h // hk, kl, d).sum(3))

        out["dv"] = shared(torch.matmul(p.transpose(-1, -2), do))
        out["dq"] = join(torch.matmul(ds, k) * scale)
        out["dk"] = shared(torch.matmul(ds.transpose(-1, -2), q) * scale)
    return out


def _plain_clip(s):
    n = s["case"]["n"]
    total = torch.zeros(n, dtype=torch.float64, device=DEV)
    for g in s["grads"]:
        g = g.float().reshape(n, -1)
        if s["case"]["shared"]:
            g = g.mean(0, keepdim=True)
        total += (g * g).sum(-1, dtype=torch.float64)
    norm = torch.sqrt(total)
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    plane = torch.zeros_like(s["plane"])
    at = 0
    for g in s["grads"]:
        k = g[0].numel()
        plane[:, at:at + k] = g.float().reshape(n, -1) * factor[:, None]
        at += -(-k // 4) * 4
    return {"norm": norm.float(), "plane": plane}


def _plain(s):
    return {"rotate": _plain_rotate, "attend": _plain_attend, "clip": _plain_clip}[s["kind"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    n, k = case["n"], case["kind"]
    if k == "clip":
        shapes = _shapes(case)
        each = [math.prod(x) for x in shapes]
        size = sum(each)
        wide = each[0] + each[-2]
        return {"bytes": n * (4 * size + 4 * (size - wide) + (2 if case["wide"] == "bf16" else 4) * wide + 4), "flops": 3 * n * size}
    b = 2 if case["dtype"] == "bf16" else 4
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    rows = n * case["seqs"] * case["q_len"]
    if k == "rotate":
        e = rows * (h + hk) * d
        # in: heads and the gradient; out: rotated heads and the gradient of what they were
        return {"bytes": e * b * (4 if case["back"] else 2) + rows * 4, "flops": e * (20 if case["back"] else 8)}
    first, end, _ = _key_ranges(case, 0)
    pairs = int((end - first).clamp(min=0).sum()) * h
    if case["mask"] == "cache":
        keys = int((end.amax(-1) - first.amin(-1)).clamp(min=0).sum())
    else:
        keys = n * case["seqs"] * case["kv_len"]
    # out and, with gradients, dout, dq, dk, dv
    return {"bytes": (rows * h * d * (4 if case["back"] else 2) + keys * hk * d * (4 if case["back"] else 2)) * b, "flops": pairs * d * (14 if case["back"] else 4)}


# ---- 64 bits ----------------------------------------------------------------------------------------
def _exact_rotate(s):
    c = s["case"]
    n, h, d, rows, r = c["n"], c["heads"], c["d"], c["seqs"] * c["q_len"], c["rotated"]
    turn = torch.polar(torch.ones_like(s["freq"]), torch.zeros_like(s["freq"])) if r else None
    out, dqk, dgain = [], [], []
    for i in range(n):
        x = s["qk"][i].double().view(rows, -1, d)
        gain = torch.cat([s["q_gain"][i].double().repeat(h, 1), s["k_gain"][i].double().repeat(c["kv_heads"], 1)])
        rstd = 1.0 / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS)
        if not c["norm"]:
            gain, rstd = torch.ones_like(gain), torch.ones_like(rstd)
        if r:
            angle = torch.outer(s["pos"][i].double(), s["freq"])
            turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]

        def rotated(v, by):
            if not r:
                return v
            both = v[..., :r].reshape(rows, -1, r // 2, 2) if c["paired"] else torch.stack(v[..., :r].chunk(2, -1), -1)
            z = torch.view_as_real(torch.view_as_complex(both.contiguous()) * by)
            z = z.reshape(rows, -1, r) if c["paired"] else torch.cat((z[..., 0], z[..., 1]), -1)
            return torch.cat((z, v[..., r:]), -1)

        out.append(rotated(x * rstd * gain, turn).reshape(rows, -1))
        if c["back"]:
            t = rotated(s["dout"][i].double().view(rows, -1, d), turn.conj() if r else None)
            dot = (t * gain * x).sum(-1, keepdim=True)
            dqk.append((t * gain * rstd - (x * dot * rstd ** 3 / d if c["norm"] else 0.0)).reshape(rows, -1))
            dgain.append((t * x * rstd).sum(0))
    got = {"out": torch.stack(out)}
    if c["back"]:
        got["dqk"] = torch.stack(dqk)
        if c["norm"]:
            dgain = torch.stack(dgain)
            got.update(dq_gain=dgain[:, :h].sum(1), dk_gain=dgain[:, h:].sum(1))
    return got


def _exact_attend(s):
    c = s["case"]
    n, b, ql, kl, h, hk, d = (c[k] for k in ("n", "seqs", "q_len", "kv_len", "heads", "kv_heads", "d"))
    f64 = dict(dtype=torch.float64, device=DEV)
    got = {"out": torch.zeros(n, b, ql, h, d, **f64)}
    if c["back"]:
        got.update(dq=torch.zeros(n, b, ql, h, d, **f64), dk=torch.zeros(n, b, kl, hk, d, **f64), dv=torch.zeros(n, b, kl, hk, d, **f64))
    j = torch.arange(kl, device=DEV)
    # several sequences and heads at a time
    some = max(1, 200_000_000 // (ql * kl * h))
    for r in range(n):
        for b0 in range(0, b, some):
            at = slice(b0, min(b, b0 + some))
            q = s["q"][r].view(b, ql, hk, h // hk, d)[at].double().permute(2, 3, 0, 1, 4)
            k, v = (s[x][r].view(b, kl, hk, d)[at].double().permute(2, 0, 1, 3) for x in ("k", "v"))
            first, end, pos = (s[x][r].view(b, ql, 1)[at] for x in ("first", "end", "pos"))
            seen = (j >= first) & (j < end)
            for kh in range(hk):
                kt = k[kh].transpose(1, 2).contiguous()
                for g in range(h // hk):
                    head = kh * (h // hk) + g
                    raw = torch.bmm(q[kh, g].contiguous(), kt) / math.sqrt(d)
                    z, slope = raw, None
                    if c["cap"]:
                        z = torch.tanh(raw / c["cap"]) * c["cap"]
                        slope = 1.0 - (z / c["cap"]).square()
                    if c["slopes"]:
                        z = z - s["slopes"][r, head].double() * (pos - j).abs().double()
                    z = z.masked_fill(~seen, float("-inf"))
                    lse = torch.logsumexp(z, -1, keepdim=True)
                    p = torch.exp(z - lse.clamp(min=-1e300)).masked_fill(~seen, 0.0)
                    del z, raw
                    o = torch.bmm(p, v[kh].contiguous())
                    got["out"][r, at, :, head] = o
                    if not c["back"]:
                        continue
                    do = s["dout"][r].view(b, ql, h, d)[at, :, head].double()
                    dp = torch.bmm(do.contiguous(), v[kh].transpose(1, 2).contiguous())
                    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
                    if slope is not None:
                        ds = ds * slope
                    ds = ds / math.sqrt(d)
                    got["dv"][r, at, :, kh] += torch.bmm(p.transpose(1, 2).contiguous(), do.contiguous())
                    got["dq"][r, at, :, head] = torch.bmm(ds, k[kh].contiguous())
                    got["dk"][r, at, :, kh] += torch.bmm(ds.transpose(1, 2).contiguous(), q[kh, g].contiguous())
                    del p, dp, ds
    return {key: x.reshape(n, -1, x.shape[-2] * d) for key, x in got.items()}


def _exact_clip(s):
    n = s["case"]["n"]
    squares = [0.0] * n
    for g in s["grads"]:
        mean = sum(g[r].double() for r in range(n)) / n if s["case"]["shared"] else None
        for r in range(n):
            squares[r] = squares[r] + (g[r].double() if mean is None else mean).square().sum()
    norm = torch.stack([torch.sqrt(x) for x in squares])
    plane = torch.zeros(s["plane"].shape, dtype=torch.float64, device=DEV)
    for r in range(n):
        factor = min(1.0, s["max_norm"] / float(norm[r]))
        at = 0
        for g in s["grads"]:
            x = g[r].double().flatten()
            plane[r, at:at + x.numel()] = x * factor
            at += (x.numel() + 3) // 4 * 4
    return {"norm": norm, "plane": plane}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend, "clip": _exact_clip}[case["kind"]](s)
