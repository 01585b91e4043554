"""Rows whose label names no class take no part in the output layer's gradients, whatever their row of h holds."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H
import test_lm_ops_vocab as V

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


# h as it is given, copied for its width, and through memory; contractions whole and in pieces
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,width,classes,piece", [(2, 90, 72, 1032, 0), (2, 90, 75, 1032, 256), (2, 270, 72, 8200, 0), (1, 270, 333, 8200, 2048), (1, 1900, 264, 2304, 0)])
def test_what_a_row_that_does_not_count_holds(n, rows, width, classes, piece, dtype):
    h, w, bias, labels = V.make(n, rows, width, classes, 8)
    for i, (label, value) in enumerate([(-1, float("nan")), (classes, float("inf")), (2 ** 31 - 1, -float("inf")), (-100, float("nan"))]):
        labels[:, 3 + 7 * i] = label
        h[:, 3 + 7 * i, i::3] = value
    out = V.call(h, w, bias, labels, dtype, piece)
    assert all(torch.all(torch.isfinite(t)) for t in out)
    zeroed = h.clone()
    zeroed[(labels < 0) | (labels >= classes)] = 0
    same = V.call(zeroed, w, bias, labels, dtype, piece)
    assert all(torch.equal(a, b) for a, b in zip(out, same))
    V.check(out, zeroed, w, bias, labels)
    loss, mean = V.call(h, w, bias, labels, dtype, piece, only_loss=True)
    assert torch.all(torch.isfinite(loss)) and torch.all(torch.isfinite(mean))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("classes", [1000, 8200])
@pytest.mark.parametrize("pad,rep,off", [(8, 64, 8), (1, 3, 1)])
def test_in_rows_of_other_strides(pad, rep, off, classes, dtype):
    n, rows, width = 2, 130, 264
    h, w, bias, labels = V.make(n, rows, width, classes, 9)
    labels[:, 5::9] = -1
    want = V.call(h, w, bias, labels, dtype, 0)
    h[labels < 0] = float("nan")
    got = V.call(R.strided(h, pad, rep, off), w, bias, labels, dtype, 0)
    assert all(torch.all(torch.isfinite(t)) for t in got)
    if off == 8:                      # the same products on the same values
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    h[labels < 0] = 0
    V.check(got, h, w, bias, labels)
