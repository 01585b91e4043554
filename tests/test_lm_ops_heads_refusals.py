"""Argument checks of the rotation, attention and gradient-norm operators, and their structures' layout.  No GPU needed: every call here is refused before anything is
enqueued (the addresses are made up), or asks for a size."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

import paper_2604_24708_amd as H
from paper_2604_24708_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 40            # an aligned address that nothing reads
NAN = float("nan")


def rows(row, rep, dev=P):
    return B.hdet_rows(dev, row, rep)


def fill(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def rotary(**kw):
    a = B.hdet_rotary_args(n_replicas=2, dtype=H.HDET_TYPE_BF16, rows=3, head_dim=16, q_heads=4, k_heads=2, rotated=8, eps=1e-6, magnitude=1.0, q_gain_dev=P,
                           q_gain_stride=16, k_gain_dev=P, k_gain_stride=16, positions_dev=P, freq_dev=P)
    a.q, a.k, a.q_out, a.k_out = rows(64, 192), rows(32, 96), rows(64, 192), rows(32, 96)
    return fill(a, kw)


def rotary_grad(**kw):
    a = B.hdet_rotary_grad_args(n_replicas=2, dtype=H.HDET_TYPE_F32, rows=3, head_dim=16, q_heads=4, k_heads=2, rotated=8, eps=1e-6, magnitude=1.0, q_gain_dev=P,
                                q_gain_stride=16, k_gain_dev=P, k_gain_stride=16, positions_dev=P, freq_dev=P, dq_gain_dev=P, dq_gain_stride=16, dk_gain_dev=P,
                                dk_gain_stride=16, workspace_dev=P, workspace_bytes=1 << 20)
    a.q, a.dq_out, a.dq = rows(64, 192), rows(64, 192), rows(64, 192)
    a.k, a.dk_out, a.dk = rows(32, 96), rows(32, 96), rows(32, 96)
    return fill(a, kw)


def attention(**kw):
    a = B.hdet_attention_args(n_replicas=2, dtype=H.HDET_TYPE_BF16, seqs=2, q_len=3, kv_len=5, heads=4, kv_heads=2, head_dim=16, causal=1, scale=0.25, lse_dev=P,
                              slopes_dev=P, slopes_stride=4, positions_dev=P, first_dev=P, end_dev=P, workspace_dev=P, workspace_bytes=1 << 30)
    a.q, a.out, a.k, a.v = rows(64, 384), rows(64, 384, 2 * P), rows(32, 320), rows(32, 320)
    return fill(a, kw)


def attention_grad(**kw):
    a = B.hdet_attention_grad_args(n_replicas=2, dtype=H.HDET_TYPE_F32, seqs=2, q_len=3, kv_len=5, heads=4, kv_heads=2, head_dim=16, causal=1, scale=0.25, lse_dev=P,
                                   slopes_dev=P, slopes_stride=4, workspace_dev=P, workspace_bytes=1 << 30)
    a.q = a.out = a.dout = rows(64, 384)
    a.k = a.v = rows(32, 320)
    a.dq, a.dk, a.dv = rows(64, 384, 2 * P), rows(32, 320, 3 * P), rows(32, 320, 4 * P)
    return fill(a, kw)


def clip(tensors=None, **kw):
    items = tensors if tensors is not None else [tensor()]
    held = (B.hdet_grad_tensor * max(len(items), 1))(*items)
    a = B.hdet_clip_args(n_replicas=2, n_tensors=len(items), tensors_host=held, max_norm=1.0, norm_dev=P, workspace_dev=P, workspace_bytes=1 << 30)
    return fill(a, kw)


def tensor(**kw):
    return fill(B.hdet_grad_tensor(rows(7, 21), rows(7, 21, P + 4096), 3, 7, H.HDET_TYPE_F32), kw)


SIZES = [dict(n_replicas=0), dict(n_replicas=65), dict(seqs=-1), dict(q_len=-1), dict(kv_len=-1), dict(seqs=1 << 12, q_len=1 << 10), dict(kv_len=1 << 28), dict(heads=0),
         dict(heads=5), dict(kv_heads=0), dict(kv_heads=-2), dict(head_dim=0), dict(head_dim=129), dict(heads=1 << 17, kv_heads=1 << 16), dict(dtype=2), dict(window=-1),
         dict(scale=NAN), dict(scale=float("inf")), dict(softcap=-1.0), dict(softcap=NAN), dict(q=rows(64, 384, None)), dict(q=rows(63, 384)), dict(q=rows(64, 384, P + 1)),
         dict(k=rows(32, 320, None)), dict(k=rows(31, 320)), dict(v=rows(32, 320, None)), dict(v=rows(-32, 320)), dict(slopes_dev=P + 2), dict(slopes_stride=-1),
         dict(positions_dev=P + 1), dict(first_dev=P + 2), dict(end_dev=P + 3)]
HEADS = [dict(n_replicas=0), dict(n_replicas=65), dict(rows=-1), dict(rows=(1 << 21) + 1), dict(dtype=3), dict(head_dim=0), dict(head_dim=257), dict(q_heads=0),
         dict(q_heads=1 << 17), dict(k_heads=0), dict(rotated=7), dict(rotated=-2), dict(rotated=18), dict(layout=2), dict(period=-1), dict(eps=-1.0), dict(eps=NAN),
         dict(magnitude=NAN), dict(magnitude=float("inf")), dict(freq_dev=None), dict(freq_dev=P + 4), dict(positions_dev=P + 2), dict(q_gain_dev=P + 1),
         dict(q_gain_stride=-1), dict(k_gain_stride=-1)]
BAD = [
    ("hdet_head_rotary", rotary, HEADS + [dict(q=rows(64, 192, None)), dict(q=rows(63, 192)), dict(q_out=rows(64, 192, None)), dict(q_out=rows(64, 100)), dict(k_out=rows(32, 96, None)),
                                          dict(k_out=rows(31, 96)), dict(k=rows(32, 96, P + 1))]),
    ("hdet_head_rotary_backward", rotary_grad, HEADS + [
        dict(q=rows(64, 192, None)), dict(k=rows(32, 96, None)), dict(dq_out=rows(64, 192, None)), dict(dk_out=rows(32, 96, None)), dict(dq=rows(64, 192, None)),
        dict(dk=rows(32, 96, None)), dict(dq=rows(64, 128)), dict(q_gain_dev=None), dict(k_gain_dev=None), dict(dq_gain_stride=15), dict(dk_gain_stride=15),
        dict(workspace_dev=None), dict(workspace_bytes=100), dict(workspace_dev=P + 8)]),
    ("hdet_attention", attention, SIZES + [dict(out=rows(64, 384, None)), dict(out=rows(64, 200, 2 * P)), dict(lse_dev=P + 2), dict(out=rows(64, 384))]),
    ("hdet_attention_backward", attention_grad, SIZES + [
        dict(out=rows(64, 384, None)), dict(dout=rows(64, 384, None)), dict(lse_dev=None), dict(dq=rows(64, 384, None)), dict(dk=rows(32, 320, None)),
        dict(dv=rows(32, 320, None)), dict(dk=rows(32, 200, 3 * P)), dict(dv=rows(30, 320, 4 * P)), dict(dq=rows(64, 384)), dict(dv=rows(32, 320)), dict(dv=rows(32, 320, 3 * P)), dict(workspace_bytes=0), dict(workspace_dev=None), dict(workspace_dev=P + 4)]),
    ("hdet_clip_gradients", clip, [
        dict(n_replicas=0), dict(n_replicas=65), dict(n_tensors=-1), dict(n_tensors=H.HDET_MAX_GRAD_TENSORS + 1), dict(tensors_host=None), dict(grad_mode=2),
        dict(max_norm=-1.0), dict(max_norm=NAN), dict(norm_dev=None), dict(norm_dev=P + 2), dict(workspace_bytes=0), dict(workspace_dev=None), dict(workspace_dev=P + 8),
        dict(tensors=[tensor(dtype=2)]), dict(tensors=[tensor(rows=-1)]), dict(tensors=[tensor(width=-1)]), dict(tensors=[tensor(rows=1 << 40)]),
        dict(tensors=[tensor(grad=rows(7, 21, None))]), dict(tensors=[tensor(grad=rows(6, 21))]), dict(tensors=[tensor(out=rows(7, 14))]),
        dict(tensors=[tensor(out=rows(7, 0, None), grad=rows(7, 0))]), dict(tensors=[tensor(out=rows(7, 21, P + 2))]), dict(tensors=[tensor(), tensor()]),
        dict(tensors=[tensor(out=rows(0, 0, None)), tensor(out=rows(0, 0, None))]), dict(tensors=[tensor(out=rows(0, 0, None)), tensor(out=rows(7, 21, P))])]),
]


@pytest.mark.parametrize("name,make,bad", [(n, m, b) for n, m, bs in BAD for b in bs], ids=lambda v: None if callable(v) else str(v)[:40])
def test_refused(name, make, bad):
    a = make(**bad)
    with pytest.raises(H.HdetError) as e:
        B._check(getattr(H.load_library(), name)(C.byref(a), None))
    assert e.value.code == H.HDET_EINVAL
    assert name in H.hdet_last_error() and len(H.hdet_last_error()) > len(name) + 5


@pytest.mark.parametrize("name", [n for n, _, _ in BAD])
def test_null_arguments(name):
    assert getattr(H.load_library(), name)(None, None) == H.HDET_EINVAL


def test_workspace_sizes():
    assert H.hdet_head_rotary_backward_workspace(2, 0, 64, 4, 2) == 0
    assert H.hdet_head_rotary_backward_workspace(2, 1000, 64, 4, 2) >= 2 * 2 * 64 * 4
    # a training step's forward pass needs none; few queries over many keys leave no more than a few results for each
    assert H.hdet_attention_workspace(8, 16, 512, 512, 16, 4, 64) == 0
    assert H.hdet_attention_workspace(1, 1, 1, 1 << 20, 8, 1, 128) <= 64 << 20
    assert H.hdet_attention_backward_workspace(2, 3, 100, 50, 4, 2, 64) >= 2 * 3 * 100 * 4 * 4
    assert H.hdet_attention_backward_workspace(2, 3, 0, 50, 4, 2, 64) == 0
    assert H.hdet_clip_gradients_workspace(8, 5) > 0
    for call in [lambda: H.hdet_head_rotary_backward_workspace(0, 1, 1, 1), lambda: H.hdet_head_rotary_backward_workspace(1, 1, 0, 1),
                 lambda: H.hdet_head_rotary_backward_workspace(1, 1, 1, 0), lambda: H.hdet_attention_workspace(1, 1, 1, 1, 3, 2, 8),
                 lambda: H.hdet_attention_workspace(1, -1, 1, 1, 2, 2, 8), lambda: H.hdet_attention_backward_workspace(1, 1, 1, 1, 2, 2, 0),
                 lambda: H.hdet_clip_gradients_workspace(0, 1), lambda: H.hdet_clip_gradients_workspace(1, -1)]:
        with pytest.raises(H.HdetError) as e:
            call()
        assert e.value.code == H.HDET_EINVAL


def test_binding_refuses_what_the_library_cannot_see():
    q, k = torch.zeros(2, 6, 64), torch.zeros(2, 6, 32)
    freq = torch.zeros(8, dtype=torch.float64)
    for call in [lambda: H.hdet_head_rotary(q, q, 16),                                        # host memory
                 lambda: H.hdet_head_rotary(q, q, 15),                                        # no whole heads
                 lambda: H.hdet_head_rotary(q.half(), q, 16), lambda: H.hdet_head_rotary(q, q, 0),
                 lambda: H.hdet_attention(q, k, k, q, 4, 2, 2), lambda: H.hdet_attention(q, k, k, q, 5, 1, 2), lambda: H.hdet_attention(q, k, k, q, 4, 2, 4),
                 lambda: H.hdet_attention(q, k, k, q, 4, 2, 0), lambda: H.hdet_attention(q, k, k, q, 0, 2, 1),
                 lambda: H.hdet_gradient_list([q]), lambda: H.hdet_gradient_list([q, k], [q]), lambda: H.hdet_gradient_list([q[0, 0]]),
                 lambda: H.hdet_gradient_list([q, torch.zeros(3, 6, 32)]), lambda: H.hdet_head_rotary(q, q, 16, freq=freq)]:
        with pytest.raises(ValueError):
            call()


def test_tensors_on_another_device_are_refused(monkeypatch):
    class Tensor:
        def __init__(self, device):
            self.device = torch.device("cuda", device)

        def get_device(self):
            return self.device.index

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    B._on_current_device(q=Tensor(1), k=None, v=Tensor(1))
    with pytest.raises(ValueError, match="v is on cuda:0, the current device is cuda:1"):
        B._on_current_device(q=Tensor(1), k=None, v=Tensor(0))


def test_structures_have_the_c_compilers_layout():
    names = ["hdet_rotary_args", "hdet_rotary_grad_args", "hdet_attention_args", "hdet_attention_grad_args", "hdet_grad_tensor", "hdet_clip_args"]
    lines, want = [], []
    for n in names:
        t = getattr(B, n)
        lines.append(f'printf("%zu ", sizeof({n}));')
        want.append(C.sizeof(t))
        for f, _ in t._fields_:
            lines.append(f'printf("%zu ", offsetof({n}, {f}));')
            want.append(getattr(t, f).offset)
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "hdet.h"\nint main(void) {' + "\n".join(lines) + "return 0; }"
    with tempfile.TemporaryDirectory() as d:
        c = os.path.join(d, "s.c")
        open(c, "w").write(src)
        exe = os.path.join(d, "s")
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe], check=True)
        got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == want
