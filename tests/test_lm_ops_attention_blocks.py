"""hdet_attention where it takes blocks of 128 queries (calls of few blocks divide the keys instead): every kind of mask and score, tiles across ranges' ends, numbers that are not finite, maxima
that rise late, and the orders of few and of many blocks; forward and backward, against 64 bits."""
import math

import pytest
import torch

import heads_reference as R
from test_lm_ops_attention import BF16, DEV, F32, backward, forward, inputs, ints, packed

pytestmark = pytest.mark.gpu

# replicas, sequences, queries, keys, heads, key heads, columns
SIZES = {
    "short": (16, 1, 200, 200, 8, 8, 24), "shared": (4, 4, 333, 333, 8, 4, 64), "wide": (16, 1, 600, 600, 8, 8, 128), "longer keys": (8, 2, 300, 1500, 16, 4, 64),
    "long keys": (8, 1, 520, 2100, 16, 16, 128), "odd": (6, 3, 257, 311, 9, 3, 50), "odd and wide": (6, 3, 257, 311, 9, 3, 100),
}
# blocks in the order of their lengths, of a number of heads that the chip's 8 parts divide and of another; in the heads' order, the same two
ORDERS = {"longest first": (8, 2, 300, 300, 8, 8, 16), "longest first, odd": (5, 3, 300, 300, 23, 23, 16), "by heads": (64, 4, 200, 200, 16, 4, 32), "by heads, odd": (63, 3, 150, 150, 11, 11, 16)}
each = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
sizes = pytest.mark.parametrize("size", list(SIZES))


def make(size, dtype, seed=0):
    n, seqs, q_len, kv_len, heads, kv_heads, d = {**SIZES, **ORDERS}[size]
    return inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=seed + d), (heads, kv_heads, seqs)


def run_and_check(q, k, v, dout, heads, kv_heads, seqs, back=True, **how):
    """As everywhere, and 2^-126 for every term of a sum, times what stands beside p in it: the exponential gives 0 for what is below fp32's normal numbers (far keys under slopes: p of 10^-40)."""
    out, lse = forward(q, k, v, heads, kv_heads, seqs, **how)
    want = R.attention(q, k, v, heads, kv_heads, seqs, dout if back else None, **how)
    tiny, d = 2.0 ** -126, q.shape[2] // heads
    q_max, k_max, v_max, do_max = (float(x.float().nan_to_num(0.0, 0.0, 0.0).abs().max()) for x in (q, k, v, dout))
    keys, rows, scale = k.shape[1] // seqs, q.shape[1] // seqs * (heads // kv_heads), abs(how.get("scale", d ** -0.5))
    dz = 2.0 * d * do_max * v_max                               # dp - dot
    R.check(out, want["out"], want["bound_out"] + tiny * keys * v_max, "out")
    R.check(lse, want["lse"], want["bound_lse"], "lse")
    if back:
        floor = {"dq": keys * dz * k_max * scale, "dk": rows * dz * q_max * scale, "dv": rows * do_max}
        for name, x in zip(("dq", "dk", "dv"), backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, **how)):
            R.check(x, want[name], want["bound_" + name] + tiny * floor[name], name)
    return out, lse


def test_the_sizes_take_blocks_of_queries():
    """By the names of the kernels that run."""
    from torch.profiler import ProfilerActivity, profile
    for size, sizes_ in {**SIZES, **ORDERS}.items():
        for dtype in (BF16, F32):
            (q, k, v, _), how = make(size, dtype)
            with profile(activities=[ProfilerActivity.CUDA]) as p:
                forward(q, k, v, *how)
                forward(q, k, v, *how, window=40)
                torch.cuda.synchronize()
            names = [e.key for e in p.key_averages() if "attend_" in e.key]
            if not names:
                pytest.skip("the profiler names no kernels here")
            assert len(names) == 1 and "attend_kernel<" in names[0], (size, names)


@each
@sizes
@pytest.mark.parametrize("how", [dict(), dict(causal=False), dict(window=1), dict(window=70), dict(window=64, causal=False), dict(softcap=2.0), dict(softcap=30.0, causal=False, window=100),
                                 dict(scale=-0.3), dict(scale=0.0)], ids=str)
def test_scores(size, how, dtype):
    (q, k, v, dout), shape = make(size, dtype)
    run_and_check(q, k, v, dout, *shape, **how)


@each
@sizes
def test_slopes(size, dtype):
    (q, k, v, dout), shape = make(size, dtype, seed=1)
    g = torch.Generator(device=DEV).manual_seed(1)
    slopes = torch.rand(q.shape[0], shape[0], generator=g, device=DEV) * 0.3
    run_and_check(q, k, v, dout, *shape, slopes=slopes)
    positions = torch.randint(-50, 2 * k.shape[1], q.shape[:2], generator=g, device=DEV, dtype=torch.int32)
    run_and_check(q, k, v, dout, *shape, slopes=slopes, causal=False, softcap=3.0, positions=positions)


@each
@sizes
def test_documents_prefixes_and_ranges(size, dtype):
    (q, k, v, dout), shape = make(size, dtype, seed=2)
    n, seqs, q_len, kv_len = SIZES[size][:4]
    first, end = packed(n, seqs, q_len, kv_len)
    run_and_check(q, k, v, dout, *shape, causal=False, first=first, end=end.clamp(max=kv_len))
    run_and_check(q, k, v, dout, *shape, causal=True, window=33, first=first, softcap=10.0)
    end = torch.clamp(torch.arange(q_len, dtype=torch.int32).repeat(n, seqs) + 1, min=100)
    end[:, -37:] = 0
    run_and_check(q, k, v, dout, *shape, causal=False, end=ints(end))
    g = torch.Generator().manual_seed(9)
    lo = torch.randint(-50, kv_len + 20, (n, seqs * q_len), generator=g)
    run_and_check(q, k, v, dout, *shape, causal=False, first=ints(lo), end=ints(lo + torch.randint(-10, 300, lo.shape, generator=g)))


@each
@pytest.mark.parametrize("size", list(ORDERS))
def test_orders_of_blocks(size, dtype):
    (q, k, v, dout), shape = make(size, dtype, seed=3)
    run_and_check(q, k, v, dout, *shape)
    n, seqs, q_len = ORDERS[size][:3]
    first, end = packed(n, seqs, q_len, 4)
    run_and_check(q, k, v, dout, *shape, causal=False, first=first, end=end, softcap=20.0)


@each
@sizes
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf], ids=str)
def test_what_nothing_attends_leaves_no_trace(size, bad, dtype):
    (q, k, v, dout), shape = make(size, dtype, seed=4)
    n, seqs, q_len, kv_len = SIZES[size][:4]
    at = torch.arange(q_len).repeat(seqs)
    # keys 50 .. 59 and queries 100 .. 109 of each sequence take part in nothing; keys from 130 on are room that nobody has written
    lo, hi = torch.where(at >= 60, 60, 0), torch.where(at < 60, torch.clamp(at + 1, max=50), torch.clamp(at + 1, max=130))
    hi[(at >= 100) & (at < 110)] = 0
    key = torch.arange(kv_len).repeat(seqs)
    keys, rows = ((key >= 50) & (key < 60)) | (key >= 130), (at >= 100) & (at < 110)
    k[:, keys], v[:, keys], q[:, rows], dout[:, rows] = bad, bad, bad, bad
    how = dict(causal=False, first=ints(lo.expand(n, -1).contiguous()), end=ints(hi.expand(n, -1).contiguous()))
    out, lse = run_and_check(q, k, v, dout, *shape, **how)
    assert all(bool(torch.isfinite(x).all()) for x in (out, *backward(q, k, v, out, lse, dout, *shape, **how)))


@each
@sizes
def test_an_infinite_value_reaches_its_column_alone(size, dtype):
    (q, k, v, _), (heads, kv_heads, seqs) = make(size, dtype, seed=5)
    n, _, q_len, kv_len, _, _, d = SIZES[size]
    clean = v.clone()
    v.view(n, seqs, kv_len, kv_heads, d)[:, :, 70, 0, 3] = math.inf
    clean.view(n, seqs, kv_len, kv_heads, d)[:, :, 70, 0, 3] = 0.0
    out, lse = forward(q, k, v, heads, kv_heads, seqs)
    want = R.attention(q, k, clean, heads, kv_heads, seqs)
    reached = torch.zeros_like(out, dtype=torch.bool)
    from_row = max(0, 70 - (kv_len - q_len))
    reached.view(n, seqs, q_len, heads, d)[:, :, from_row:, :heads // kv_heads, 3] = True
    R.check(torch.where(reached, torch.zeros_like(out), out), want["out"].masked_fill(reached, 0.0), want["bound_out"], "out")
    R.check(lse, want["lse"], want["bound_lse"], "lse")
    assert bool((out[reached] == math.inf).all())


@each
@sizes
def test_maxima_that_rise_late(size, dtype):
    """Scores of +-10^4, a maximum that rises from tile to tile by far more than fp32's exponentials hold, and one that falls."""
    (q, k, v, dout), shape = make(size, dtype, seed=6)
    n, seqs, q_len, kv_len, heads, kv_heads, d = SIZES[size]
    ramp = torch.linspace(0.0, 3.0, kv_len, device=DEV).repeat(seqs)[None, :, None]
    for sign in (1.0, -1.0):
        run_and_check(q * 0 + 2.0, (k.float() * 0.1 + sign * ramp).to(dtype), v, dout, *shape, causal=sign < 0)
    run_and_check(q * 16, k * 8, v, dout, *shape, back=False)
    run_and_check(q * 16, k * 8, v, dout, *shape, back=False, softcap=500.0)
    # one key of every 32 from the 128th on is ahead of all others by 2^126.96
    q.zero_().view(n, -1, heads, d)[..., 0] = 1.0
    k.zero_().view(n, seqs, kv_len, kv_heads, d)[:, :, 128::32, :, 0] = 88.0
    run_and_check(q, k, v, dout, *shape, back=False, scale=1.0, causal=False)
