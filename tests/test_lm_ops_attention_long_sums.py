"""Sums over many keys in fp32: how far results are from 64 bits does not grow with the number of keys.

An addition is off by 2^-24 / sqrt(3) (times 0.72, a mantissa's mean) of the running sum, 2.5e-8; a sum of L values of either sign has come to sqrt(k / L) of itself after k of them, so that all L
additions are off by 2.5e-8 sqrt(L / 2): 5.7e-7 in runs of 1024 keys, whatever their number, 1.7e-6 in one sum of 9000.  p is off by 3e-7 (a score of some sums of 64 products, and its difference to lse),
dz by 6e-7 (p, a row dot and another sum of products): out by 6.4e-7, dq by 8.3e-7; in one sum by 1.7e-6 and 1.8e-6.  A quarter of these is allowed on top."""
import pytest
import torch

import heads_reference as R
from test_lm_ops_attention import DEV, F32, backward, distance, forward, inputs

pytestmark = pytest.mark.gpu


def definition(q, k, v, dout, heads, slopes):
    """out, lse and dq of one replica and one sequence, every query at position 0 over all keys, head by head in 64 bits."""
    d, scale = q.shape[1] // heads, (q.shape[1] // heads) ** -0.5
    out, dq, lse = torch.empty_like(q, dtype=torch.float64), torch.empty_like(q, dtype=torch.float64), torch.empty(heads, q.shape[0], dtype=torch.float64, device=DEV)
    for h in range(heads):
        c = slice(h * d, h * d + d)
        qh, kh, vh, do = (x[:, c].double() for x in (q, k, v, dout))
        z = torch.matmul(qh, kh.t().contiguous()) * scale - float(slopes[0, h]) * torch.arange(k.shape[0], device=DEV)
        lse[h] = torch.logsumexp(z, -1)
        p = torch.exp(z - lse[h][:, None])
        out[:, c] = torch.matmul(p, vh)
        dz = p * (torch.matmul(do, vh.t().contiguous()) - (do * out[:, c]).sum(-1, keepdim=True))
        dq[:, c] = torch.matmul(dz, kh) * scale
    return out, lse, dq


def run_and_check(n, q_len, kv_len, heads, d, back, slope=0.0):
    """Replicas share their keys (a replica stride of 0); the first of them is compared."""
    q, _, _, dout = inputs(n, 1, q_len, 1, heads, heads, d, F32, seed=d)
    _, k, v, _ = inputs(1, 1, 1, kv_len, heads, heads, d, F32, seed=d + 1)
    shared = [x.expand(n, -1, -1) for x in (k, v)]
    how = dict(causal=False)
    slopes = torch.full((n, heads), slope, device=DEV)
    if slope:
        how.update(slopes=slopes, positions=torch.zeros(n, q_len, dtype=torch.int32, device=DEV))
    out, lse = forward(q, *shared, heads, heads, 1, **how)
    want = definition(q[0], k[0], v[0], dout[0], heads, slopes)
    assert distance(out[0], want[0]) <= 0.8e-6
    assert float((lse[0].double() - want[1]).abs().max()) <= 4e-6          # (five of its own roundings, 2^-24 of 10 to 16, for the largest of thousands)
    if back:
        grads = [torch.empty_like(q), *(torch.empty(n, kv_len, heads * d, device=DEV) for _ in range(2))]
        dq = backward(q, *shared, out, lse, dout, heads, heads, 1, grads=grads, **how)[0]
        assert distance(dq[0], want[2]) <= 1.05e-6


@pytest.mark.parametrize("d", [64, 128, 50])
def test_blocks_of_queries(d):
    """1024 blocks of 128 queries and more: no walk over the keys is divided."""
    run_and_check(16, 512, 9000, 16, d, back=True)


@pytest.mark.parametrize("d,kv_len", [(64, 36000), (128, 18000), (41, 36000)])
def test_few_queries(d, kv_len):
    """512 blocks of few queries: the wavefronts of one block divide the keys, 9000 to each."""
    run_and_check(64, 16, kv_len, 8, d, back=False)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_fall_with_the_distance(d):
    """The reference of the exponentials follows the maximum all the way; 9000 keys of weights that fall by a factor of 1.25 altogether."""
    run_and_check(16, 512, 9000, 16, d, back=True, slope=2.0 ** -15 * 0.8)
    run_and_check(64, 16, 36000 if d == 64 else 18000, 8, d, back=False, slope=2.0 ** -16)
