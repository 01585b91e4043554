"""The output layer with its loss at sizes whose logits stay in the matrix cores' registers: more than 8192 classes, or more than a tile of 256 x 256 on every fourth
compute unit.  Bounds as in test_lm_ops_vocab."""
import pytest
import torch

import ops_reference as R
import test_lm_ops_vocab as V

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

SHAPES = [(1, 1, 64, 8200, 0), (1, 3, 8, 9001, 0), (2, 40, 72, 8194, 2048), (1, 300, 264, 9003, 0), (1, 257, 777, 8500, 4096), (3, 130, 200, 10000, 256), (1, 1100, 520, 12345, 0),
          (4, 520, 136, 2600, 0), (2, 2050, 256, 2051, 1024), (1, 4100, 96, 1300, 0), (8, 256, 330, 2304, 768)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,width,classes,piece", SHAPES)
def test_loss_and_gradients(n, rows, width, classes, piece, dtype):
    V.test_loss_and_gradients(n, rows, width, classes, piece, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("width,piece", [(72, 0), (333, 2048)])
def test_rows_that_do_not_count(width, piece, dtype):
    n, rows, classes = 3, 270, 8200
    h, w, bias, labels = V.make(n, rows, width, classes, 1)
    labels[0] = -1
    labels[1] = classes                                     # in the padding of the last tile of classes
    labels[1, 5] = classes - 1
    labels[2, ::3] = 2 ** 31 - 1
    h[2, 0] = float("nan")
    out = V.call(h, w, bias, labels, dtype, piece)
    assert torch.all(out[0][0] == 0) and float(out[1][0]) == 0
    for t in out[2:]:
        assert torch.all(t[0] == 0)
    assert torch.all(out[2][1, :5] == 0) and torch.all(out[2][1, 6:] == 0) and bool((out[2][1, 5] != 0).any())
    assert torch.all(out[0][2, ::3] == 0) and torch.all(torch.isfinite(out[0])) and torch.all(torch.isfinite(out[4])) and torch.all(out[2][2, 0] == 0)
    h[2, 0] = 0
    V.check(V.call(h, w, bias, labels, dtype, piece), h, w, bias, labels)


@pytest.mark.parametrize("width", [40, 300])
@pytest.mark.parametrize("piece", [0, 2560])
def test_masked_classes_and_a_bad_row(width, piece):
    n, rows, classes = 1, 60, 9000
    h, w, bias, labels = V.make(n, rows, width, classes, 2, ignored=0.0)
    bias[0, :6000] = -float("inf")                          # whole tiles, and whole pieces of classes
    labels.copy_(6000 + labels % (classes - 6000))
    out = V.call(h, w, bias, labels, F32, piece)
    ref = R.vocab_loss(h, w[:, 6000:], bias[:, 6000:], labels - 6000)
    assert torch.all((out[0].double() - ref[0]).abs() <= 1e-5 * (1 + ref[0].abs()))
    assert torch.all(out[3][:, :6000] == 0) and torch.all(out[4][:, :6000] == 0)
    assert R.rel(out[3][:, 6000:], ref[3]) <= 1e-5 and R.rel(out[2], ref[2]) <= 2 * 2.0 ** -9
    h[0, 7, 3] = float("nan")                               # a row that counts: its loss and gradient are lost, the other rows' are not
    out = V.call(h, w, bias, labels, BF, piece)
    assert torch.isnan(out[0][0, 7]) and torch.all(torch.isnan(out[2][0, 7]))
    assert int(torch.isnan(out[0]).sum()) == 1 and int(torch.isnan(out[2]).any(-1).sum()) == 1


@pytest.mark.parametrize("size", [30.0, 300.0])
def test_large_logits(size):
    h, w, bias, labels = V.make(1, 64, 256, 9000, 3, spread=size)
    V.check(V.call(h, w, bias, labels, F32, 2048), h, w, bias, labels)


def test_columns_of_very_different_sizes():
    """An fp32 dw holds its columns' own precision: columns of h between 2^-40 and 2^20 of one another."""
    h, w, bias, labels = V.make(2, 400, 136, 9000, 9)
    e = torch.linspace(-40, 20, 136, device=R.DEV).round()
    h = (h.double() * torch.exp2(e)).to(BF)
    w = (w.double() * torch.exp2(-e.clamp(min=0))).to(BF)
    out = V.call(h, w, bias, labels, F32, 0)
    want = R.vocab_loss(h, w, bias, labels)[3]
    err = (out[3].double() - want).norm(dim=1) / want.norm(dim=1)
    L = (136 + 2) * R.U * float(torch.matmul(h.double().abs(), w.double().abs().transpose(1, 2).contiguous()).max()) + 64 * R.U
    assert float(err.max()) <= 2e-6 + 4 * L


def test_gradient_against_differences():
    V.test_gradient_against_differences(256, 8456)
