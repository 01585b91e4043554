"""hdet_attention and its backward pass against 64 bits: head sizes and groups, lengths from none to long ones, masks, strides, non-finite numbers in places that
nothing attends, captured graphs and streams."""
import pytest
import torch

import heads_reference as R
import ops_reference as O
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=0, size=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(rows, width, std=1.0):
        return (torch.randn(n, rows, width, generator=g, device=DEV) * std).to(dtype)

    return [normal(seqs * q_len, heads * d, size), normal(seqs * kv_len, kv_heads * d), normal(seqs * kv_len, kv_heads * d), normal(seqs * q_len, heads * d)]


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32, device=DEV)


def forward(q, k, v, heads, kv_heads, seqs, out=None, stream=None, work=None, **how):
    n, rows, width = q.shape
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full((n, heads, rows), 7.0, device=DEV)
    if work is None:
        size = H.hdet_attention_workspace(n, seqs, rows // seqs, k.shape[1] // seqs, heads, kv_heads, width // heads)
        work = torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)
    H.hdet_attention(q, k, v, out, heads, kv_heads, seqs, lse=lse, workspace=work, stream=stream, **how)
    return out, lse


def backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, grads=None, stream=None, work=None, **how):
    n, rows, width = q.shape
    dq, dk, dv = grads or [torch.full_like(x, 7.0) for x in (q, k, v)]
    if work is None:
        size = H.hdet_attention_backward_workspace(n, seqs, rows // seqs, k.shape[1] // seqs, heads, kv_heads, width // heads)
        work = torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)
    H.hdet_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, heads, kv_heads, seqs, workspace=work, stream=stream, **how)
    return dq, dk, dv


def run_and_check(q, k, v, dout, heads, kv_heads, seqs, back=True, **how):
    out, lse = forward(q, k, v, heads, kv_heads, seqs, **how)
    want = R.attention(q, k, v, heads, kv_heads, seqs, dout if back else None, **how)
    R.check(out, want["out"], want["bound_out"], "out")
    R.check(lse, want["lse"], want["bound_lse"], "lse")
    if back:
        for name, x in zip(("dq", "dk", "dv"), backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, **how)):
            R.check(x, want[name], want["bound_" + name], name)
    return out, lse


# ---- sizes --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,seqs,q_len,kv_len,heads,kv_heads,d", [
    (1, 1, 1, 1, 1, 1, 1), (2, 2, 1, 1, 2, 1, 64), (1, 2, 2, 2, 3, 3, 5), (2, 1, 31, 31, 2, 1, 16), (1, 2, 32, 32, 2, 2, 64), (2, 1, 33, 65, 4, 2, 72),
    (1, 1, 64, 64, 2, 1, 128), (1, 3, 65, 65, 6, 2, 80), (2, 1, 127, 130, 3, 1, 33), (1, 1, 128, 128, 2, 2, 127), (1, 2, 129, 129, 4, 4, 96), (1, 1, 200, 333, 8, 1, 64),
    (1, 1, 257, 256, 2, 1, 40), (2, 1, 300, 300, 1, 1, 7), (1, 1, 513, 640, 2, 1, 112)])
def test_sizes(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype):
    q, k, v, dout = inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=q_len + d)
    run_and_check(q, k, v, dout, heads, kv_heads, seqs)
    run_and_check(q, k, v, dout, heads, kv_heads, seqs, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 72])
def test_walks_in_parts(d, dtype):
    """Few blocks over long sequences: the backward pass's kernels divide their walks; empty rows, documents and an infinite gradient among them."""
    n, q_len = 1, 1300
    q, k, v, dout = inputs(n, 1, q_len, q_len, 2, 1, d, dtype, seed=d)
    run_and_check(q, k, v, dout, 2, 1, 1)
    run_and_check(q, k, v, dout, 2, 1, 1, causal=False, window=700, softcap=4.0)
    first, end = packed(n, 1, q_len, 5)
    run_and_check(q, k, v, dout, 2, 1, 1, causal=False, first=first, end=end)
    bad = dout.clone()
    bad[0, 1000, 5] = float("inf")
    out, lse = forward(q, k, v, 2, 1, 1)
    _, dk, dv = backward(q, k, v, out, lse, bad, 2, 1, 1)
    want = R.attention(q, k, v, 2, 1, 1, dout)
    R.check(dk[:, 1001:], want["dk"][:, 1001:], want["bound_dk"][:, 1001:], "dk")
    reached = torch.zeros_like(dv, dtype=torch.bool)
    reached[:, :1001, 5] = True
    assert bool((~torch.isfinite(dv[reached])).all()) and bool((~torch.isfinite(dk[:, :1001])).all())
    R.check(torch.where(reached, torch.zeros_like(dv), dv), want["dv"].masked_fill(reached, 0.0), want["bound_dv"], "dv")


@pytest.mark.parametrize("d", [64, 50])
def test_runs_of_rows_in_divided_walks(d):
    """fp32, more than 1024 rows to a part of a walk: the parts are made by several launches that add up."""
    q, k, v, dout = inputs(1, 1, 6200, 6200, 4, 1, d, F32, seed=d)
    run_and_check(q, k, v, dout, 4, 1, 1)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_nothing_to_do(dtype):
    # no queries: the keys' gradients are 0; no keys: every query is empty
    q, k, v, dout = inputs(2, 2, 0, 5, 4, 2, 16, dtype)
    dk, dv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    lse = torch.empty(2, 4, 0, device=DEV)
    H.hdet_attention(q, k, v, q.clone(), 4, 2, 2, lse=lse)
    H.hdet_attention_backward(q, k, v, q, lse, dout, q.clone(), dk, dv, 4, 2, 2)
    assert not dk.any() and not dv.any()
    q, k, v, dout = inputs(2, 2, 5, 0, 4, 2, 16, dtype)
    out, lse = forward(q, k, v, 4, 2, 2)
    assert not out.any() and bool((lse == float("-inf")).all())
    assert not backward(q, k, v, out, lse, dout, 4, 2, 2)[0].any()
    H.hdet_attention(q[:, :0], k, v, q[:, :0], 4, 2, 0)


def distance(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("q_len,heads,kv_heads,d", [(2, 32, 8, 96), (4, 16, 4, 32), (48, 4, 1, 64)])
def test_few_queries_of_many_heads(q_len, heads, kv_heads, d):
    """Gradients that few queries make are as far from 64 bits as their own rounding takes them: p and dz enter to 2^-16 and their errors in fp32 are 2^-20 or so, where that rounding is
    some 2^-9 (a tenth is allowed for both)."""
    q, k, v, dout = inputs(2, 2, q_len, q_len, heads, kv_heads, d, BF16, seed=d)
    out, lse = forward(q, k, v, heads, kv_heads, 2)
    want = R.attention(q, k, v, heads, kv_heads, 2, dout)
    for name, x in zip(("dk", "dv"), backward(q, k, v, out, lse, dout, heads, kv_heads, 2)[1:]):
        assert distance(x, want[name]) <= 1.1 * distance(want[name].to(BF16), want[name]), name


@pytest.mark.parametrize("d", [64, 128])
def test_short_documents_in_a_long_sequence(d):
    """dq of rows that attend one or two keys of 2100, where the walk over the keys is divided: as far from 64 bits as its own rounding takes it (a tenth is allowed for dz in two parts and
    for fp32)."""
    q_len = 2100
    q, k, v, dout = inputs(1, 1, q_len, q_len, 2, 1, d, BF16, seed=d)
    first = ints((torch.arange(q_len) // 2 * 2)[None])
    out, lse = forward(q, k, v, 2, 1, 1, first=first)
    want = R.attention(q, k, v, 2, 1, 1, dout, first=first)
    dq = backward(q, k, v, out, lse, dout, 2, 1, 1, first=first)[0]
    assert distance(dq, want["dq"]) <= 1.1 * distance(want["dq"].to(BF16), want["dq"])
    assert not dq[:, ::2].any()


@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 64), (32, 8, 128)])
def test_gradients_of_many_rows_in_fp32(heads, kv_heads, d):
    """Four heads of 1088 rows to a key.  A running sum over M rows rounds M times, each 2^-24 / sqrt(3) (times 0.72, a mantissa's mean) of a sum that the first queries, which attend few
    keys, have made as large as it gets: sqrt(M) times 2.5e-8, 8.0e-7 for runs of 1024 rows and 1.6e-6 for one sum of 4352.  p and dz are off by 6e-7 (scores, lse and dots at 2^-24 of 16)."""
    q, k, v, dout = inputs(2, 1, 1088, 1088, heads, kv_heads, d, F32, seed=d)
    out, lse = forward(q, k, v, heads, kv_heads, 1, softcap=30.0)
    want = R.attention(q, k, v, heads, kv_heads, 1, dout, softcap=30.0)
    for name, x in zip(("dk", "dv"), backward(q, k, v, out, lse, dout, heads, kv_heads, 1, softcap=30.0)[1:]):
        assert distance(x, want[name]) <= 1e-6, name


# ---- scores and masks ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("how", [dict(softcap=2.0), dict(softcap=30.0, causal=False), dict(window=1), dict(window=17), dict(window=64, causal=False), dict(window=200, softcap=5.0),
                                 dict(scale=0.0), dict(scale=-0.5), dict(scale=1.0, softcap=1.0)], ids=str)
@pytest.mark.parametrize("d", [24, 64, 128])
def test_scores(how, d, dtype):
    q, k, v, dout = inputs(2, 2, 150, 150, 4, 2, d, dtype, seed=d)
    run_and_check(q, k, v, dout, 4, 2, 2, **how)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [24, 64, 128])
def test_slopes(d, dtype):
    n, heads = 2, 6
    q, k, v, dout = inputs(n, 1, 190, 190, heads, 2, d, dtype, seed=d)
    slopes = torch.rand(n, heads, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) * 0.3
    run_and_check(q, k, v, dout, heads, 2, 1, slopes=slopes)
    run_and_check(q, k, v, dout, heads, 2, 1, slopes=slopes, causal=False, softcap=3.0, positions=ints(torch.randint(-50, 400, (n, 190))))


def packed(n, seqs, q_len, seed):
    """Ranges of packed documents, the first of a sequence 40 tokens, and up to 30 rows behind the last that attend nothing."""
    g = torch.Generator().manual_seed(seed)
    first, end = torch.zeros(n * seqs, q_len, dtype=torch.int32), torch.zeros(n * seqs, q_len, dtype=torch.int32)
    for s in range(n * seqs):
        at, last, size = 0, q_len - int(torch.randint(0, 31, (1,), generator=g)), 40
        while at < last:
            stop = min(last, at + size)
            first[s, at:stop] = at
            end[s, at:stop] = torch.arange(at, stop, dtype=torch.int32) + 1
            at, size = stop, int(torch.randint(1, 100, (1,), generator=g))
    return first.view(n, -1).to(DEV), end.view(n, -1).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [24, 64, 128])
def test_documents_and_prefixes(d, dtype):
    n, seqs, q_len = 2, 2, 310
    q, k, v, dout = inputs(n, seqs, q_len, q_len, 4, 2, d, dtype, seed=d + 1)
    first, end = packed(n, seqs, q_len, d)
    run_and_check(q, k, v, dout, 4, 2, seqs, causal=False, first=first, end=end)
    run_and_check(q, k, v, dout, 4, 2, seqs, causal=True, window=33, first=first, softcap=10.0)
    pos = torch.arange(q_len, dtype=torch.int32).repeat(n, seqs)
    prefix = torch.clamp(pos + 1, min=100)
    prefix[:, -37:] = 0
    run_and_check(q, k, v, dout, 4, 2, seqs, causal=False, end=ints(prefix))
    # ranges in no order, beyond both ends, empty ones among them
    g = torch.Generator().manual_seed(9)
    lo = torch.randint(-50, q_len + 20, (n, seqs * q_len), generator=g)
    run_and_check(q, k, v, dout, 4, 2, seqs, causal=False, first=ints(lo), end=ints(lo + torch.randint(-10, 200, lo.shape, generator=g)))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_extreme_ranges(dtype):
    """32-bit ends of positions and ranges do not wrap around."""
    q, k, v, dout = inputs(1, 1, 70, 70, 2, 1, 64, dtype)
    top, low = 2 ** 31 - 1, -2 ** 31
    for how in [dict(positions=top), dict(positions=low), dict(positions=top, window=top), dict(positions=low, window=top, causal=False), dict(first=top), dict(end=low),
                dict(first=low, end=top), dict(first=top, end=low, causal=False)]:
        how = {a: torch.full((1, 70), b, dtype=torch.int32, device=DEV) if a in ("positions", "first", "end") else b for a, b in how.items()}
        run_and_check(q, k, v, dout, 2, 1, 1, **how)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=str)
def test_what_nothing_attends_leaves_no_trace(bad, d, dtype):
    n, seqs, q_len = 1, 2, 140
    q, k, v, dout = inputs(n, seqs, q_len, q_len, 4, 2, d, dtype, seed=3)
    pos = torch.arange(q_len).repeat(seqs)
    # keys 50 .. 59 of each sequence, and queries 100 .. 109, take part in nothing; keys from 130 on are room that nobody has written
    lo, hi = torch.where(pos >= 60, 60, 0), torch.where(pos < 60, torch.clamp(pos + 1, max=50), torch.clamp(pos + 1, max=130))
    hi[(pos >= 100) & (pos < 110)] = 0
    first, end = ints(lo[None]), ints(hi[None])
    keys = ((pos >= 50) & (pos < 60)) | (pos >= 130)
    rows = (pos >= 100) & (pos < 110)
    k[:, keys], v[:, keys], q[:, rows], dout[:, rows] = bad, bad, bad, bad
    how = dict(causal=False, first=first, end=end)
    out, lse = run_and_check(q, k, v, dout, 4, 2, seqs, **how)
    grads = backward(q, k, v, out, lse, dout, 4, 2, seqs, **how)
    assert all(bool(torch.isfinite(x).all()) for x in (out, *grads))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 64, 128])
def test_a_later_token_that_is_not_finite(d, dtype):
    """With causal masks rows before a NaN token stay as they were, in the forward and in the backward pass."""
    q, k, v, dout = inputs(1, 1, 150, 150, 2, 1, d, dtype, seed=4)
    want = R.attention(q, k, v, 2, 1, 1, dout)
    at = 77
    for x in (q, k, v):
        x[:, at] = float("nan")
    out, lse = forward(q, k, v, 2, 1, 1)
    R.check(out[:, :at], want["out"][:, :at], want["bound_out"][:, :at], "out")
    R.check(lse[..., :at], want["lse"][..., :at], want["bound_lse"][..., :at], "lse")
    assert bool(torch.isnan(out[:, at:]).all())
    dq, _, _ = backward(q, k, v, out, lse, dout, 2, 1, 1)
    R.check(dq[:, :at], want["dq"][:, :at], want["bound_dq"][:, :at], "dq")
    assert bool(torch.isnan(dq[:, at:]).all())
    # a NaN in one query and its gradient reaches the keys that it attends and no others
    q, k, v, dout = inputs(1, 1, 150, 150, 2, 1, d, dtype, seed=4)
    q2, dout2 = q.clone(), dout.clone()
    q2[:, at] = float("nan")
    dout2[:, at] = float("nan")
    out2, lse2 = forward(q2, k, v, 2, 1, 1)
    _, dk, dv = backward(q2, k, v, out2, lse2, dout2, 2, 1, 1)
    assert bool(torch.isnan(dk[:, :at + 1]).all()) and bool(torch.isnan(dv[:, :at + 1]).all())
    R.check(dk[:, at + 1:], want["dk"][:, at + 1:], want["bound_dk"][:, at + 1:], "dk")
    R.check(dv[:, at + 1:], want["dv"][:, at + 1:], want["bound_dv"][:, at + 1:], "dv")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_an_infinite_value_reaches_its_column_alone(d, dtype):
    q, k, v, _ = inputs(1, 1, 150, 150, 2, 1, d, dtype, seed=5)
    v[:, 70, 3] = float("inf")
    out, _ = forward(q, k, v, 2, 1, 1)
    clean = v.clone()
    clean[:, 70, 3] = 0
    want = R.attention(q, k, clean, 2, 1, 1)
    reached = torch.zeros_like(out, dtype=torch.bool)
    reached[:, 70:, [3, 3 + d]] = True
    R.check(torch.where(reached, torch.zeros_like(out), out), want["out"].masked_fill(reached, 0.0), want["bound_out"], "out")
    assert bool((out[reached] == float("inf")).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_large_and_far_scores(dtype):
    """Scores of +-10^4, rows that see only very low ones, a maximum that rises from tile to tile."""
    q, k, v, dout = inputs(1, 1, 260, 260, 2, 1, 64, dtype, seed=6)
    ramp = torch.linspace(0.0, 3.0, 260, device=DEV)[None, :, None]
    run_and_check(q * 0 + 2.0, (k.float() * 0.1 + ramp).to(dtype), v, dout, 2, 1, 1, causal=False)
    run_and_check(q * 0 + 2.0, (k.float() * 0.1 - ramp).to(dtype), v, dout, 2, 1, 1)
    run_and_check(q * 16, k * 8, v, dout, 2, 1, 1, back=False)
    slopes = torch.full((1, 2), 1000.0, device=DEV)
    run_and_check(q, k, v, dout, 2, 1, 1, back=False, causal=False, slopes=slopes, positions=ints(torch.full((1, 260), 2 ** 20)))


# ---- one token and a few over a long cache ------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,seqs,q_len,kv_len,heads,kv_heads,d", [
    (1, 1, 1, 5000, 1, 1, 64), (2, 3, 1, 1000, 8, 2, 64), (1, 2, 1, 4097, 16, 1, 128), (2, 1, 5, 3001, 6, 2, 80), (1, 1, 3, 20000, 4, 4, 16), (1, 1, 40, 6000, 2, 2, 128),
    (2, 16, 1, 130, 32, 8, 64), (1, 1, 7, 2500, 9, 3, 41)])
def test_few_queries_over_many_keys(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype):
    q, k, v, dout = inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=kv_len)
    run_and_check(q, k, v, dout, heads, kv_heads, seqs, back=False, causal=False)
    g = torch.Generator().manual_seed(2)
    start = torch.randint(0, kv_len - q_len, (n, seqs, 1), generator=g)
    start[0, 0] = 0
    pos = ints((start + torch.arange(q_len)).view(n, -1))
    # room behind what the sequences have
    run_and_check(q, k, v, dout, heads, kv_heads, seqs, back=False, positions=pos)
    run_and_check(q, k, v, dout, heads, kv_heads, seqs, back=False, positions=pos, window=97, softcap=20.0, slopes=torch.full((n, heads), 0.01, device=DEV))
    none = pos.clone()
    none[:, 0] = -1                      # a query that attends nothing
    run_and_check(q, k, v, dout, heads, kv_heads, seqs, back=False, positions=none)


@pytest.mark.parametrize("kv_len", [256, 8192])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_late_scores_that_nearly_leave_the_range(dtype, kv_len):
    """One key of every 32 from the 128th on is ahead of all others by 2^126.96: exponentials relative to the first keys are in fp32's range, their sum is not."""
    q, k, v, _ = inputs(1, 1, 1, kv_len, 1, 1, 16, dtype, seed=5)
    q.zero_()[..., 0] = 1.0
    k.zero_()[:, 128::32, 0] = 88.0
    run_and_check(q, k, v, None, 1, 1, 1, back=False, scale=1.0, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_a_cache_with_room_that_nobody_has_written(dtype):
    n, seqs, kv_len = 2, 2, 3000
    q, k, v, _ = inputs(n, seqs, 1, kv_len, 8, 2, 64, dtype, seed=8)
    end = ints([[700, 2999], [1, 0]])
    for r in range(n):
        for b in range(seqs):
            for x in (k, v):
                x[r, b * kv_len + int(end[r, b]):(b + 1) * kv_len] = float("nan")
    out, lse = run_and_check(q, k, v, None, 8, 2, seqs, back=False, causal=False, end=end)
    assert bool(torch.isfinite(out).all()) and not out[1, 1].any()


# ---- memory -------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("row_pad,rep_pad,offset", [(8, 0, 0), (3, 5, 1), (64, 24, 8), (1, 0, 0)])
def test_strides_and_what_lies_between(row_pad, rep_pad, offset, dtype):
    n, seqs, q_len, heads, kv_heads, d = 2, 2, 100, 4, 2, 64
    q, k, v, dout = inputs(n, seqs, q_len, q_len, heads, kv_heads, d, dtype, seed=11)
    how = dict(row_pad=row_pad, rep_pad=rep_pad, offset=offset)
    sq, sk, sv, sd = (O.strided(x, **how) for x in (q, k, v, dout))
    out = O.strided(torch.zeros_like(q), **how)
    grads = [O.strided(torch.zeros_like(x), **how) for x in (q, k, v)]
    _, lse = forward(sq, sk, sv, heads, kv_heads, seqs, out=out)
    backward(sq, sk, sv, out, lse, sd, heads, kv_heads, seqs, grads=grads)
    want = R.attention(q, k, v, heads, kv_heads, seqs, dout)
    for name, x in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        R.check(x, want[name], want["bound_" + name], name)
        base = x._base if x._base is not None else x
        inside = torch.zeros_like(base, dtype=torch.bool)
        torch.as_strided(inside, x.shape, x.stride(), x.storage_offset()).fill_(True)
        assert bool(torch.isnan(base[~inside].float()).all())          # the gaps are as they were


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_slices_of_one_matrix_and_replicas_between_each_other(dtype):
    n, q_len, heads, kv_heads, d = 2, 130, 4, 2, 64
    wide = (heads + 2 * kv_heads) * d
    # [token][replica][q | k | v]
    store = torch.randn(q_len, n, wide, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(dtype)
    qkv, grads = store.transpose(0, 1), torch.zeros_like(store).transpose(0, 1)
    cut = [slice(0, heads * d), slice(heads * d, (heads + kv_heads) * d), slice((heads + kv_heads) * d, wide)]
    q, k, v = (qkv[..., c] for c in cut)
    dout = torch.randn(n, q_len, heads * d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(dtype)
    out, lse = forward(q, k, v, heads, kv_heads, 1)
    backward(q, k, v, out, lse, dout, heads, kv_heads, 1, grads=[grads[..., c] for c in cut])
    want = R.attention(q.contiguous(), k.contiguous(), v.contiguous(), heads, kv_heads, 1, dout)
    R.check(out, want["out"], want["bound_out"], "out")
    for name, c in zip(("dq", "dk", "dv"), cut):
        R.check(grads[..., c], want[name], want["bound_" + name], name)


def test_replicas_that_share_their_keys():
    """A replica stride of 0 among the inputs."""
    q, k, v, _ = inputs(3, 1, 70, 70, 2, 1, 64, BF16)
    k, v = k[:1].expand(3, -1, -1), v[:1].expand(3, -1, -1)
    run_and_check(q, k, v, None, 2, 1, 1, back=False)


@pytest.mark.parametrize("d,q_len,kv_len", [(64, 1, 600000), (128, 40, 300000)])
def test_offsets_beyond_32_bits(d, q_len, kv_len):
    """A cache of more than 2^32 bytes in a replica; what is attended lies at its end."""
    seqs, kv_heads, heads = 16, 8, 8
    k = torch.zeros(1, seqs * kv_len, kv_heads * d, dtype=BF16, device=DEV)
    v = torch.zeros_like(k)
    assert k.numel() * 2 > 2 ** 32
    q, tail_k, tail_v, _ = inputs(1, seqs, q_len, 200, heads, kv_heads, d, BF16, seed=13)
    at = (torch.arange(seqs, device=DEV)[:, None] * kv_len + kv_len - 200 + torch.arange(200, device=DEV)).flatten()
    k[:, at], v[:, at] = tail_k, tail_v
    first = torch.full((1, seqs * q_len), kv_len - 200, dtype=torch.int32, device=DEV)
    out, lse = forward(q, k, v, heads, kv_heads, seqs, causal=False, first=first)
    want = R.attention(q, tail_k, tail_v, heads, kv_heads, seqs, causal=False)
    R.check(out, want["out"], want["bound_out"], "out")
    R.check(lse, want["lse"], want["bound_lse"], "lse")
    whole, _ = forward(q, k, v, heads, kv_heads, seqs, causal=False)
    # all the others have score 0 and value 0
    weight = torch.exp(want["lse"].double()) / (torch.exp(want["lse"].double()) + (kv_len - 200))
    scaled = want["out"].view(1, seqs * q_len, heads, d) * weight.transpose(1, 2)[..., None]
    bound = (want["bound_out"] * 2).view_as(scaled) * weight.transpose(1, 2)[..., None] + 2.0 ** -8 * scaled.abs() + R.U * kv_len ** 0.5 * scaled.abs()
    R.check(whole, scaled.reshape(whole.shape), bound.reshape(whole.shape) + 1e-9, "out over all keys")


# ---- graphs and streams -------------------------------------------------------------------------
@pytest.mark.parametrize("q_len,kv_len", [(130, 130), (1, 3000)])
def test_captured_and_replayed(q_len, kv_len):
    """Two graphs that share a workspace, replayed in turn with eager calls between them."""
    n, seqs, heads, kv_heads, d = 2, 2, 4, 2, 64
    sets = [inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, BF16, seed=s) for s in (1, 2)]
    size = max(H.hdet_attention_workspace(n, seqs, q_len, kv_len, heads, kv_heads, d), H.hdet_attention_backward_workspace(n, seqs, q_len, kv_len, heads, kv_heads, d))
    work = torch.zeros(max(size, 16), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    graphs, results = [], []
    for q, k, v, dout in sets:
        out, lse, grads = torch.empty_like(q), torch.empty(n, heads, seqs * q_len, device=DEV), [torch.empty_like(x) for x in (q, k, v)]

        def step():
            H.hdet_attention(q, k, v, out, heads, kv_heads, seqs, lse=lse, workspace=work, stream=torch.cuda.current_stream().cuda_stream)
            H.hdet_attention_backward(q, k, v, out, lse, dout, *grads, heads, kv_heads, seqs, workspace=work, stream=torch.cuda.current_stream().cuda_stream)

        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
        results.append((out, lse, *grads))
    for turn in range(3):
        for i, (q, k, v, dout) in enumerate(sets):
            for x in results[i]:
                x.fill_(float("nan"))
            q.normal_(generator=torch.Generator(device=DEV).manual_seed(10 * turn + i))
            graphs[i].replay()
            torch.cuda.synchronize()
            out, lse = forward(q, k, v, heads, kv_heads, seqs)
            want = (out, lse, *backward(q, k, v, out, lse, dout, heads, kv_heads, seqs))
            assert all(torch.equal(a, b) for a, b in zip(results[i], want))


def test_two_streams_at_once():
    n, seqs, heads, kv_heads, d = 2, 2, 4, 2, 64
    jobs = []
    for i, (q_len, kv_len) in enumerate([(200, 200), (1, 5000)]):
        q, k, v, dout = inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, BF16, seed=i)
        out, lse = forward(q, k, v, heads, kv_heads, seqs)
        jobs.append((q, k, v, out.clone(), lse.clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for q, k, v, _, _, s in jobs:
            with torch.cuda.stream(s):
                got.append(forward(q, k, v, heads, kv_heads, seqs, stream=s.cuda_stream))
        torch.cuda.synchronize()
        for (out, lse), job in zip(got, jobs):
            assert torch.equal(out, job[3]) and torch.equal(lse, job[4])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_the_same_bits_every_time(dtype):
    q, k, v, dout = inputs(2, 2, 300, 300, 8, 2, 64, dtype)
    out, lse = forward(q, k, v, 8, 2, 2)
    grads = backward(q, k, v, out, lse, dout, 8, 2, 2)
    for _ in range(3):
        again = forward(q, k, v, 8, 2, 2)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
        assert all(torch.equal(a, b) for a, b in zip(backward(q, k, v, out, lse, dout, 8, 2, 2), grads))


def test_gradients_against_differences():
    """Central differences of sum(out * w) in 64 bits at fp32 inputs, against the kernels' gradients: 1e-4 in size for a step of 1e-4 and a third derivative below 10^3 or so."""
    n, seqs, q_len, heads, kv_heads, d = 1, 1, 20, 4, 2, 8
    how = dict(softcap=3.0, slopes=torch.full((n, heads), 0.1, device=DEV), window=9)
    q, k, v, dout = inputs(n, seqs, q_len, q_len, heads, kv_heads, d, F32, seed=21)
    out, lse = forward(q, k, v, heads, kv_heads, seqs, **how)
    grads = backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, **how)
    g = torch.Generator().manual_seed(3)
    for x, grad in zip((q, k, v), grads):
        for _ in range(12):
            at = (0, int(torch.randint(0, x.shape[1], (1,), generator=g)), int(torch.randint(0, x.shape[2], (1,), generator=g)))
            value = []
            for step in (1e-4, -1e-4):
                moved = [y.double() for y in (q, k, v)]
                moved[[id(q), id(k), id(v)].index(id(x))][at] += step
                value.append(float((R.attention(*moved, heads, kv_heads, seqs, **how)["out"] * dout.double()).sum()))
            assert abs((value[0] - value[1]) / 2e-4 - float(grad[at])) <= 1e-4
