"""hdet_attention's backward pass (and the forward one) on matrices whose rows lie beyond 2^32 elements and bytes of their start."""
import pytest
import torch

import heads_reference as R
from test_lm_ops_attention import BF16, DEV, F32, backward, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,pitch,q_len,d", [(BF16, 1 << 20, 4500, 64), (F32, 1 << 20, 4500, 128), (BF16, (1 << 23) + 8, 530, 128), (F32, (1 << 22) + 4, 1060, 64), (BF16, (1 << 20) + 1, 4200, 50)])
def test_rows_of_a_long_pitch(dtype, pitch, q_len, d):
    """Queries, keys, values, results and gradients are columns of the rows of two matrices of more than 2^32 elements."""
    heads, kv_heads = 4, 2
    q, k, v, dout = inputs(1, 1, q_len, q_len, heads, kv_heads, d, dtype, seed=d)
    widths = [x.shape[2] for x in (q, k, v, dout, q)]
    store, grads = (torch.full((1, q_len, pitch), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    assert store.numel() > 2 ** 32
    cut, at = [], pitch - sum(widths)
    for w in widths:
        cut.append(slice(at, at + w))
        at += w
    for c, x in zip(cut, (q, k, v, dout)):
        store[..., c] = x
    sq, sk, sv, sd, so = (store[..., c] for c in cut)
    to = [grads[..., cut[i]] for i in range(3)]
    _, lse = forward(sq, sk, sv, heads, kv_heads, 1, out=so)
    backward(sq, sk, sv, so, lse, sd, heads, kv_heads, 1, grads=to)
    want = R.attention(q, k, v, heads, kv_heads, 1, dout)
    for name, x in zip(("out", "dq", "dk", "dv"), (so, *to)):
        R.check(x, want[name], want["bound_" + name], name)
    assert bool((grads[..., : cut[0].start] == 7.0).all()) and bool((store[..., : cut[0].start] == 7.0).all()) and bool((grads[..., cut[3].start:] == 7.0).all())


@pytest.mark.parametrize("d,q_len,kv_len", [(64, 3, 600000), (128, 40, 300000)])
def test_a_cache_beyond_32_bits(d, q_len, kv_len):
    """Keys, values and their gradients of more than 2^32 bytes and elements in a replica; what is attended lies at the end of every sequence."""
    seqs, kv_heads, heads, tail = 16, 8, 8, 200
    k = torch.zeros(1, seqs * kv_len, kv_heads * d, dtype=BF16, device=DEV)
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 32
    q, tail_k, tail_v, dout = inputs(1, seqs, q_len, tail, heads, kv_heads, d, BF16, seed=13)
    at = (torch.arange(seqs, device=DEV)[:, None] * kv_len + kv_len - tail + torch.arange(tail, device=DEV)).flatten()
    k[:, at], v[:, at] = tail_k, tail_v
    first = torch.full((1, seqs * q_len), kv_len - tail, dtype=torch.int32, device=DEV)
    out, lse = forward(q, k, v, heads, kv_heads, seqs, causal=False, first=first)
    dq, dk, dv = backward(q, k, v, out, lse, dout, heads, kv_heads, seqs, causal=False, first=first)
    want = R.attention(q, tail_k, tail_v, heads, kv_heads, seqs, dout, causal=False)
    R.check(dq, want["dq"], want["bound_dq"], "dq")
    for name, x in (("dk", dk), ("dv", dv)):
        R.check(x[:, at], want[name], want["bound_" + name], name)
        x[:, at] = 0.0
        assert not x.any(), name
