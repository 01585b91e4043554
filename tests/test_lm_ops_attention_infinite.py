"""hdet_attention and its backward pass with infinite entries in queries and keys that are attended, where the definition is finite all the same: a score of minus infinity is a pair of weight 0,
one of plus or minus infinity under a cap is the cap, whose derivative is 0.  What a weight of 0 multiplies with an infinity is NaN, and nothing else is."""
import math

import pytest
import torch

import heads_reference as R
from test_lm_ops_attention import BF16, DEV, F32, backward, forward, inputs, ints, packed

pytestmark = pytest.mark.gpu


def cleaned(x):
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x))


def attention(q, k, v, heads, kv_heads, seqs, dout, scale=None, softcap=0.0, **mask):
    """The definition in 64 bits, pair by pair, over the pairs that are attended; bounds as heads_reference's, from the sizes of the finite terms (the others are in no finite sum)."""
    n, rows, width = q.shape
    d, group = width // heads, heads // kv_heads
    q_len, kv_len = rows // seqs, k.shape[1] // seqs
    scale = d ** -0.5 if scale is None else scale
    b = R.half(q.dtype) if q.dtype == BF16 else 0.0
    last = R.half(q.dtype)

    def split(x, length, count):
        return x.double().view(n, seqs, length, count, d).transpose(2, 3)

    def join(x):
        return x.transpose(2, 3).reshape(n, -1, x.shape[2] * d)

    lo, hi, _ = R.key_ranges(n, seqs, q_len, kv_len, **mask)
    j = torch.arange(kv_len, device=q.device)
    seen = ((j >= lo[..., None]) & (j < hi[..., None]))[:, :, None]
    q_, do = split(q, q_len, heads), split(dout, q_len, heads)
    k_, v_ = (split(x, kv_len, kv_heads).repeat_interleave(group, 2) for x in (k, v))

    def product(a, b):                                          # [.., i, c], [.., j, c] -> [.., i, j], terms of every pair
        return torch.stack([(a[..., i, None, :] * b).sum(-1) for i in range(a.shape[-2])], -2)

    def total(w, x):                                            # sum over j of w [.., i, j] x [.., j, c] over the attended pairs
        zero = torch.zeros((), dtype=torch.float64, device=q.device)
        return torch.stack([torch.where(seen[..., i, :, None], w[..., i, :, None] * x, zero).sum(-2) for i in range(w.shape[-2])], -2)

    def total_t(w, x):                                          # the same over i
        zero = torch.zeros((), dtype=torch.float64, device=q.device)
        return torch.stack([torch.where(seen[..., :, i, None], w[..., :, i, None] * x, zero).sum(-2) for i in range(w.shape[-1])], -2)

    z = product(q_, k_) * scale
    wide = product(cleaned(q_).abs(), cleaned(k_).abs()) * abs(scale)
    bend = torch.ones_like(z)
    if softcap:
        bend, z = 1.0 - torch.tanh(z / softcap) ** 2, softcap * torch.tanh(z / softcap)
    z = torch.where(seen, z, torch.full_like(z, -math.inf))
    some = seen.any(-1, keepdim=True)
    lse = torch.logsumexp(z, -1, keepdim=True)
    p = torch.where(some & seen, torch.exp(z - torch.where(some, lse, torch.zeros_like(lse))), torch.zeros_like(z))
    off = R.U * ((d + 16) * torch.where(seen, wide, torch.zeros_like(wide)).amax(-1, keepdim=True) + 4.0 * softcap + 4.0 * lse.abs().masked_fill(~some, 0.0) + 16.0)
    sums, rows_sum = R.U * (kv_len + 16), R.U * (q_len * group + 16)
    rel = 2.0 * off + sums + b
    o, size = total(p, v_), total(p, cleaned(v_).abs())
    dp = torch.where(seen, product(do, v_), torch.zeros_like(z))
    dp_size = product(do.abs(), cleaned(v_).abs())
    dot = torch.where(some, (do * o).sum(-1, keepdim=True), torch.zeros_like(lse))
    off_dot = (do.abs() * (rel * size + last * o.abs())).sum(-1, keepdim=True) + R.U * (d + 8) * (do.abs() * size).sum(-1, keepdim=True)
    dz = p * (dp - dot) * bend
    off_bend = 8.0 * R.U + 2.0 * off / softcap if softcap else 0.0
    off_dz = p * (off_dot + R.U * (d + 8) * dp_size) + dz.abs() * (2.0 * off + 8.0 * R.U) + p * (dp - dot).abs() * off_bend + b * dz.abs()

    def shared(x):
        return join(x.view(n, seqs, kv_heads, group, kv_len, d).sum(3))

    res = {"out": join(o), "lse": lse[..., 0].transpose(1, 2).reshape(n, heads, rows), "dq": join(total(dz, k_) * scale), "dk": shared(total_t(dz, q_) * scale), "dv": shared(total_t(p, do))}
    res["bound_out"] = join(rel * size + last * o.abs())
    res["bound_lse"] = (off + sums + 8 * R.U)[..., 0].transpose(1, 2).reshape(n, heads, rows)
    res["bound_dq"] = join(total(off_dz + sums * dz.abs(), cleaned(k_).abs()) * abs(scale)) + (last + 4 * R.U) * res["dq"].abs()
    res["bound_dk"] = shared(total_t(off_dz + rows_sum * dz.abs(), cleaned(q_).abs()) * abs(scale)) + (last + 4 * R.U) * res["dk"].abs()
    res["bound_dv"] = shared(total_t(p * (2.0 * off + rows_sum + b), do.abs())) + (last + 4 * R.U) * res["dv"].abs()
    return res


def check(got, want, name):
    """Finite where the definition is, and as near; not finite where it is not."""
    w, finite = want[name], torch.isfinite(want[name])
    R.check(torch.where(finite, got.double(), torch.zeros_like(w)), torch.where(finite, w, torch.zeros_like(w)), torch.where(finite, want["bound_" + name], torch.zeros_like(w)), name)
    assert not bool(torch.isfinite(got[~finite]).any()), f"{name}: finite where the definition is not"


def run_and_check(q, k, v, dout, heads, kv_heads, seqs, **how):
    out, lse = forward(q, k, v, heads, kv_heads, seqs, **how)
    want = attention(q, k, v, heads, kv_heads, seqs, dout, **how)
    assert bool(torch.isfinite(want["out"]).any())
    check(out, want, "out")
    check(lse, want, "lse")
    # the backward pass from the results as they are
    for name, x in zip(("dq", "dk", "dv"), backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, **how)):
        check(x, want, name)
    return want


# heads of two, three and four 32-column blocks, loose ones, groups; few queries and few keys (dk and dv in two parts), walks in parts (640 tokens of one head)
SIZES = [(1, 1, 70, 70, 2, 1, 64), (2, 1, 150, 150, 4, 2, 128), (1, 2, 130, 200, 3, 3, 40), (1, 1, 40, 290, 2, 2, 96), (1, 1, 640, 640, 1, 1, 64), (1, 1, 600, 600, 2, 1, 128),
         (16, 4, 70, 70, 8, 4, 64)]
each = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
sizes = pytest.mark.parametrize("n,seqs,q_len,kv_len,heads,kv_heads,d", SIZES)


@each
@sizes
@pytest.mark.parametrize("masks", ["all", "causal", "ranges"])
def test_keys_that_an_infinite_column_masks(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, masks):
    """A column of ones in the queries, of 0 and minus infinity in the keys: weight 0 at every third key from the second on, and at a run of keys longer than a tile."""
    q, k, v, dout = inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=d + q_len)
    at = torch.arange(kv_len, device=DEV)
    masked = ((at % 3 == 1) | ((at >= 20) & (at < 60))).repeat(seqs)
    q.view(n, -1, heads, d)[..., 5] = 1.0
    k.view(n, -1, kv_heads, d)[..., 5] = torch.where(masked, -math.inf, 0.0).to(dtype)[None, :, None]
    how = dict(causal=masks == "causal")
    if masks == "ranges":
        end = packed(n, seqs, q_len, d)[1].clamp(max=kv_len)
        how = dict(causal=False, end=torch.where(end > 0, end.clamp(min=7), end))
    want = run_and_check(q, k, v, dout, heads, kv_heads, seqs, **how)
    columns = torch.arange(heads * d, device=DEV) % d != 5
    assert bool(torch.isfinite(want["dq"][..., columns]).all()) and bool(torch.isfinite(want["dk"]).all()) and bool(torch.isfinite(want["dv"]).all())
    assert bool((want["dq"] != 0).any())


@each
@sizes
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("where", ["queries", "keys", "both"])
def test_capped_scores_of_infinite_entries(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, causal, where):
    """Scores of plus and minus the cap.  Column 3 of the queries' infinities meets keys away from 0, column 6 of the keys' the queries."""
    q, k, v, dout = inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=d + q_len + 1)
    hq, hk = q.view(n, -1, heads, d), k.view(n, -1, kv_heads, d)
    hk[..., 3] = torch.where(hk[..., 3] < 0, -1.0, 1.0).to(dtype)
    hq[..., 6] = torch.where(hq[..., 6] < 0, -1.0, 1.0).to(dtype)
    if where != "keys":
        hq[:, 11::17, :, 3] = math.inf
        hq[:, 13::29, 0, 3] = -math.inf
    if where == "keys":
        hk[:, 9::23, :, 6] = -math.inf
        hk[:, 30:64:2, 0, 6] = math.inf
    if where == "both":                                         # (an infinite query and an infinite key: minus one infinity or the other where their signs differ: NaN, in the definition too)
        hk[:, 2, 0, 6] = math.inf
    want = run_and_check(q, k, v, dout, heads, kv_heads, seqs, causal=causal, softcap=4.0)
    columns = torch.arange(heads * d, device=DEV) % d
    keys = torch.arange(kv_heads * d, device=DEV) % d
    if where != "both":
        assert bool(torch.isfinite(want["dq"][..., columns != 6]).all()) and bool(torch.isfinite(want["dk"][..., keys != 3]).all()) and bool(torch.isfinite(want["dv"]).all())
        assert bool(torch.isfinite(want["dq"]).all()) == (where == "queries") and bool(torch.isfinite(want["dk"]).all()) == (where == "keys")


@each
def test_runs_of_rows(dtype):
    """More than 1024 rows to a key (fp32: several launches that add up), infinities in the first and the last of them, a window with none of them behind it."""
    q, k, v, dout = inputs(8, 1, 420, 420, 16, 4, 64, dtype, seed=9)
    hq, hk = q.view(8, -1, 16, 64), k.view(8, -1, 4, 64)
    hk[..., 3] = torch.where(hk[..., 3] < 0, -1.0, 1.0).to(dtype)
    hq[:, 30, 0, 3] = math.inf
    hq[:, 401, 3, 3] = -math.inf
    run_and_check(q, k, v, dout, 16, 4, 1, softcap=4.0)
    want = run_and_check(q, k, v, dout, 16, 4, 1, softcap=4.0, window=100)
    assert bool(torch.isfinite(want["dk"][:, 31:301]).all())


@each
@pytest.mark.parametrize("d", [64, 128])
def test_short_documents(d, dtype):
    """Rows of few keys, whose dots are formed on a walk of their own: every document's first key is masked by an infinity, and so is what stands before it."""
    q_len = 700
    q, k, v, dout = inputs(1, 1, q_len, q_len, 2, 1, d, dtype, seed=d)
    at = torch.arange(q_len, device=DEV)
    q.view(1, -1, 2, d)[..., 5] = 1.0
    k[..., 5] = torch.where(at % 4 == 0, -math.inf, 0.0).to(dtype)
    # (a row that attends its document's first key alone has no weight at all: NaN, in the definition too)
    run_and_check(q, k, v, dout, 2, 1, 1, first=ints((at // 4 * 4)[None]), end=ints(((at + 1) * (at % 4 != 0))[None]))


@each
@pytest.mark.parametrize("q_len,heads,d", [(70, 2, 64), (3, 2, 128), (300, 16, 40)])
def test_infinite_values_and_output_gradients_of_weight_zero(q_len, heads, d, dtype):
    """An infinite value is NaN in the rows that attend it with weight 0 and infinity in the others; an infinite output gradient the same in dv."""
    n, kv_len, at = 4, 300, 40
    q, k, v, dout = inputs(n, 1, q_len, kv_len, heads, heads, d, dtype, seed=d)
    hq, hk = q.view(n, -1, heads, d), k.view(n, -1, heads, d)
    hq[..., 5] = 1.0
    hq[:, ::2, :, 5] = -1.0
    hk[..., 5] = 0.0
    hk[:, at, :, 5] = math.inf                                  # weight 0 in every other row; the rows between have a score of plus infinity and no finite results
    v.view(n, -1, heads, d)[:, at, :, 7] = math.inf
    out, lse = forward(q, k, v, heads, heads, 1, causal=False)
    rows = out.view(n, -1, heads, d)
    assert bool(torch.isnan(rows[:, 1::2]).all()) and bool(torch.isnan(rows[:, ::2, :, 7]).all())
    columns = torch.arange(d, device=DEV) != 7
    assert bool(torch.isfinite(rows[:, ::2][..., columns]).all())
    k.view(n, -1, heads, d)[:, at, :, 5] = 0.0
    out, _ = forward(q, k, v, heads, heads, 1, causal=False)
    assert bool((out.view(n, -1, heads, d)[..., 7] == math.inf).all())
    # a masked key, and an output gradient that is infinite in one row
    hk[:, at, :, 5] = math.inf
    hq[..., 5] = -1.0
    v.view(n, -1, heads, d)[:, at, :, 7] = 1.0
    dout.view(n, -1, heads, d)[:, 1, :, 9] = math.inf
    out, lse = forward(q, k, v, heads, heads, 1, causal=False)
    dv = backward(q, k, v, out, lse, dout, heads, heads, 1, causal=False)[2].view(n, -1, heads, d)
    others = torch.arange(kv_len, device=DEV) != at
    assert bool(torch.isnan(dv[:, at, :, 9]).all()) and bool((dv[:, others][..., 9] == math.inf).all())
    assert bool(torch.isfinite(dv[..., torch.arange(d, device=DEV) != 9]).all())


@each
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf], ids=str)
@pytest.mark.parametrize("n,seqs,q_len,kv_len,heads,kv_heads,d", [(1, 1, 40, 8, 2, 1, 64), (2, 2, 70, 70, 4, 2, 40), (16, 2, 300, 200, 8, 8, 128), (1, 1, 700, 700, 1, 1, 64)])
def test_rows_that_attend_nothing_beside_rows_of_such_keys_alone(n, seqs, q_len, kv_len, heads, kv_heads, d, bad, dtype):
    """Every row that attends anything has no finite results (a NaN, or weight 0 or an infinite score for all its keys); the others' are 0 all the same."""
    q, k, v, dout = inputs(n, seqs, q_len, kv_len, heads, kv_heads, d, dtype, seed=d)
    q.view(n, -1, heads, d)[..., 5] = 1.0
    k.view(n, -1, kv_heads, d)[..., 5] = bad
    at = torch.arange(q_len, device=DEV).repeat(seqs)
    end = ints(torch.where(at % 3 == 1, 0, kv_len).expand(n, -1))
    out, lse = forward(q, k, v, heads, kv_heads, seqs, causal=False, end=end)
    dq, dk, dv = backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, causal=False, end=end)
    empty = at % 3 == 1
    assert not out[:, empty].any() and bool((lse[..., empty] == -math.inf).all()) and not dq[:, empty].any()
    assert all(bool(torch.isnan(x).all()) for x in (out[:, ~empty], dq[:, ~empty], dk, dv))
