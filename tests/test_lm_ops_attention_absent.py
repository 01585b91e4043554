"""hdet_attention and its backward pass without the matrices that they do not need: no keys, no queries."""
import ctypes as C

import pytest
import torch

import paper_2604_24708_amd as H
from paper_2604_24708_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rows(x):
    return B.hdet_rows(x.data_ptr(), x.stride(1), x.stride(0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,seqs,q_len,heads,kv_heads,d", [(2, 2, 5, 4, 2, 16), (2, 3, 200, 4, 4, 64), (1, 1, 1, 1, 1, 128), (1, 2, 130, 3, 1, 41)])
def test_no_keys(n, seqs, q_len, heads, kv_heads, d, dtype):
    """Queries that attend nothing are not read: out is 0, lse minus infinity, dq 0, and q, k, v, out and dout may be absent."""
    out, dq = (torch.full((n, seqs * q_len, heads * d), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    lse = torch.full((n, heads, seqs * q_len), 7.0, device=DEV)
    work = torch.zeros(H.hdet_attention_backward_workspace(n, seqs, q_len, 0, heads, kv_heads, d) + 16, dtype=torch.uint8, device=DEV)
    sizes = dict(n_replicas=n, dtype=H.HDET_TYPE_BF16 if dtype == torch.bfloat16 else H.HDET_TYPE_F32, seqs=seqs, q_len=q_len, kv_len=0, heads=heads, kv_heads=kv_heads, head_dim=d, causal=1,
                 scale=1.0, workspace_dev=work.data_ptr(), workspace_bytes=work.numel())
    a = B.hdet_attention_args(**sizes, out=rows(out), lse_dev=lse.data_ptr())
    B._check(H.load_library().hdet_attention(C.byref(a), None))
    g = B.hdet_attention_grad_args(**sizes, dq=rows(dq))
    B._check(H.load_library().hdet_attention_backward(C.byref(g), None))
    assert not out.any() and bool((lse == float("-inf")).all()) and not dq.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,seqs,kv_len,heads,kv_heads,d", [(2, 2, 5, 4, 2, 16), (1, 3, 300, 4, 4, 64), (1, 1, 1, 1, 1, 128)])
def test_no_queries(n, seqs, kv_len, heads, kv_heads, d, dtype):
    """Keys that no query attends: dk and dv are 0, and nothing else need be there."""
    dk, dv = (torch.full((n, seqs * kv_len, kv_heads * d), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    sizes = dict(n_replicas=n, dtype=H.HDET_TYPE_BF16 if dtype == torch.bfloat16 else H.HDET_TYPE_F32, seqs=seqs, q_len=0, kv_len=kv_len, heads=heads, kv_heads=kv_heads, head_dim=d, causal=1,
                 scale=1.0)
    B._check(H.load_library().hdet_attention(C.byref(B.hdet_attention_args(**sizes)), None))
    g = B.hdet_attention_grad_args(**sizes, dk=rows(dk), dv=rows(dv))
    B._check(H.load_library().hdet_attention_backward(C.byref(g), None))
    assert not dk.any() and not dv.any()
