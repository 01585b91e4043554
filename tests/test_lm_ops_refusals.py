"""Argument checks of the language-model operators, and their structures' layout.  No GPU needed: every call here is refused before
anything is enqueued (the addresses are made up), or asks for a size."""
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


def rows(row, rep, dev=P):
    return B.hdet_rows(dev, row, rep)


def norm(**kw):
    a = B.hdet_norm_args(n_replicas=2, dtype=H.HDET_TYPE_BF16, rows=3, width=40, eps=1e-5, scale_dev=P, rstd_dev=P, gain_dev=P, gain_stride=40)
    a.x = a.resid = a.total = a.y = rows(40, 120)
    a.codes = rows(48, 144)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def norm_grad(**kw):
    a = B.hdet_norm_grad_args(n_replicas=2, dtype=H.HDET_TYPE_F32, rows=3, width=40, rstd_dev=P, gain_dev=P, gain_stride=40, dgain_dev=P, dgain_stride=40,
                              workspace_dev=P, workspace_bytes=1 << 20)
    a.total = a.dy = a.dtotal = a.dx = rows(40, 120)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def codes(**kw):
    a = B.hdet_codes_args(n_replicas=2, dtype=H.HDET_TYPE_F32, rows=3, width=40, scale_dev=P)
    a.values, a.codes = rows(40, 120), rows(48, 144)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def linear(**kw):
    a = B.hdet_linear_args(n_replicas=2, y_dtype=H.HDET_TYPE_F32, rows=3, d_in=40, d_out=7, scale_dev=P, w_scale_dev=P, bias_dev=P, bias_stride=7)
    a.codes, a.w_codes, a.y = rows(48, 144), rows(48, 336), rows(7, 21)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def linear_grad(**kw):
    a = B.hdet_linear_grad_args(n_replicas=2, rows=3, d_in=40, d_out=7, scale_dev=P, w_scale_dev=P, db_dev=P, db_stride=7, workspace_dev=P,
                                workspace_bytes=1 << 30)
    a.dy, a.codes, a.w_codes, a.dx, a.dw = rows(7, 21), rows(48, 144), rows(48, 336), rows(40, 120), rows(40, 280)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def vocab(**kw):
    a = B.hdet_vocab_args(n_replicas=2, dw_dtype=H.HDET_TYPE_F32, rows=3, width=40, classes=9, bias_dev=P, bias_stride=9, labels_dev=P, row_loss_dev=P,
                          mean_loss_dev=P, db_dev=P, db_stride=9, workspace_dev=P, workspace_bytes=1 << 30)
    a.h, a.w, a.dh, a.dw = rows(40, 120), rows(40, 360), rows(40, 120), rows(40, 360)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD = [
    ("hdet_rmsnorm", norm, [
        dict(n_replicas=0), dict(n_replicas=65), dict(rows=-1), dict(rows=(1 << 21) + 1), dict(width=0), dict(width=H.HDET_MAX_NORM_WIDTH + 1), dict(dtype=2),
        dict(eps=-1.0), dict(eps=float("nan")), dict(x=rows(40, 120, None)), dict(x=rows(40, 120, P + 1)), dict(x=rows(39, 120)), dict(x=rows(-40, 120)),
        dict(total=rows(40, 80)), dict(y=rows(39, 120)), dict(codes=rows(40, 144)), dict(codes=rows(32, 144)), dict(codes=rows(48, 144, P + 8)),
        dict(codes=rows(48, 136)), dict(scale_dev=None), dict(rstd_dev=P + 2), dict(gain_dev=None), dict(gain_stride=-1)]),
    ("hdet_rmsnorm_backward", norm_grad, [
        dict(n_replicas=0), dict(rows=-1), dict(width=0), dict(dtype=-1), dict(total=rows(40, 120, None)), dict(dy=rows(40, 120, None)),
        dict(dx=rows(40, 120, None)), dict(dx=rows(40, 0)), dict(rstd_dev=None), dict(gain_dev=None), dict(dgain_stride=39), dict(workspace_dev=None),
        dict(workspace_bytes=319), dict(workspace_dev=P + 4)]),
    ("hdet_quantise_rows", codes, [
        dict(n_replicas=0), dict(width=H.HDET_MAX_NORM_WIDTH + 1), dict(dtype=7), dict(values=rows(40, 120, None)), dict(codes=rows(48, 144, None)),
        dict(codes=rows(48, 96)), dict(scale_dev=None)]),
    ("hdet_restore_rows", codes, [
        dict(width=H.HDET_MAX_CODES_WIDTH + 1), dict(values=rows(40, 80)), dict(codes=rows(47, 144)), dict(codes=rows(1 << 22, 1 << 30)), dict(scale_dev=None)]),
    ("hdet_quantised_linear", linear, [
        dict(n_replicas=65), dict(rows=-1), dict(d_in=0), dict(d_in=H.HDET_MAX_CODES_WIDTH + 1), dict(d_out=0), dict(y_dtype=3), dict(codes=rows(48, 144, None)),
        dict(w_codes=rows(48, 336, None)), dict(scale_dev=None), dict(w_scale_dev=None), dict(y=rows(7, 21, None)), dict(y=rows(6, 21)), dict(y=rows(7, 14)),
        dict(bias_stride=-1), dict(w_codes=rows(40, 336))]),
    ("hdet_quantised_linear_backward", linear_grad, [
        dict(d_out=0), dict(dy=rows(7, 21, None)), dict(codes=rows(48, 144, None)), dict(w_codes=rows(48, 336, None)), dict(dx=rows(40, 80)), dict(dw=rows(39, 280)),
        dict(db_stride=6), dict(workspace_bytes=100), dict(workspace_dev=None)]),
    ("hdet_vocab_loss", vocab, [
        dict(n_replicas=0), dict(rows=-1), dict(width=0), dict(classes=0), dict(dw_dtype=2), dict(piece=-1), dict(h=rows(40, 120, None)), dict(w=rows(40, 360, None)),
        dict(labels_dev=None), dict(row_loss_dev=None), dict(mean_loss_dev=None), dict(dh=rows(40, 100)), dict(dw=rows(30, 360)), dict(db_stride=8),
        dict(workspace_bytes=0), dict(h=rows(40, 120, P + 1))]),
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
    assert H.hdet_rmsnorm_backward_workspace(2, 0, 64) == 0
    assert H.hdet_rmsnorm_backward_workspace(2, 1000, 64) >= 2 * 64 * 4
    assert H.hdet_quantised_linear_backward_workspace(3, 100, 33, 50) >= 3 * (100 + 50) * 40 * 2
    whole = H.hdet_vocab_loss_workspace(2, 100, 64, 5000, dw=torch.bfloat16, piece=5000)
    part = H.hdet_vocab_loss_workspace(2, 100, 64, 5000, dw=torch.bfloat16, piece=512)
    assert part < whole < H.hdet_vocab_loss_workspace(2, 100, 64, 5000, dw=torch.float32, piece=5000)
    # a large head: far less than its logits' gradient alone would take
    assert H.hdet_vocab_loss_workspace(8, 8192, 1024, 128000, dw=torch.bfloat16) < 8 * 8192 * 128000 * 2 // 8
    for call in [lambda: H.hdet_rmsnorm_backward_workspace(0, 1, 1), lambda: H.hdet_rmsnorm_backward_workspace(1, 1, 0),
                 lambda: H.hdet_quantised_linear_backward_workspace(1, -1, 1, 1), lambda: H.hdet_vocab_loss_workspace(1, 1, 1, 0),
                 lambda: H.hdet_vocab_loss_workspace(1, 1, 1, 1, piece=-5)]:
        with pytest.raises(H.HdetError) as e:
            call()
        assert e.value.code == H.HDET_EINVAL


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(2, 3, 40)
    gain = torch.ones(2, 40)
    with pytest.raises(ValueError):
        H.hdet_rmsnorm(x, gain, y=torch.zeros_like(x))                    # host memory
    with pytest.raises(ValueError):
        H.hdet_rmsnorm(x.half(), gain, y=torch.zeros_like(x))             # a type that is not taken
    with pytest.raises(ValueError):
        H.hdet_quantise_rows(x, torch.zeros(2, 3, 40, dtype=torch.int8), torch.zeros(2, 3))
    c = H.hdet_codes_empty(2, 3, 40, device="cpu")
    assert c.shape == (2, 3, 40) and c.stride() == (144, 48, 1)


def test_structures_have_the_c_compilers_layout():
    names = ["hdet_rows", "hdet_norm_args", "hdet_norm_grad_args", "hdet_codes_args", "hdet_linear_args", "hdet_linear_grad_args", "hdet_vocab_args"]
    lines = []
    want = []
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
