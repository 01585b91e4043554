"""Row losses where exponentials say all but nothing: logits that are whole numbers, far apart."""
import pytest
import torch

import ops_reference as R
import test_lm_ops_vocab as V

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

TOPS = [3008.0, 304.0, -304.0, 40.0, -1984.0, 96.0, 1024.0, 0.0]
GAP = 64.0


@pytest.mark.parametrize("only_loss", [False, True])
@pytest.mark.parametrize("classes,piece", [(300, 0), (300, 64), (9000, 0), (9000, 2048)])
def test_rows_certain_of_their_label(classes, piece, only_loss):
    """Row r's logits are exact: TOPS[r % 8] at one class, 64 less at the others.  The loss is that of sums of numbers next to 1 (one rounding of an argument below 1/2, 2^-25;
    one of the exponential, 2^-23; a few of fp32 sums, 2^-24 each, of which all but one term are below 2^-90): within 2^-22, and its own rounding.  The logits' size is in none of
    them, so a row of 3008 is as exact as one of 0, and none has a loss below that of certainty."""
    rows, width = 64, 8
    g = torch.Generator().manual_seed(classes)
    h = torch.zeros(1, rows, width)
    h[0, torch.arange(rows), torch.arange(rows) % width] = 1.0
    top = torch.randint(0, classes, (width,), generator=g)
    tops = torch.tensor(TOPS)
    w = (tops - GAP).expand(classes, width).clone()
    w[top, torch.arange(width)] = tops
    labels = torch.where(torch.arange(rows) % 16 < 12, top[torch.arange(rows) % width], (top[torch.arange(rows) % width] + 1) % classes).to(torch.int32)[None]
    h, w, labels = h.to(BF).to(R.DEV), w[None].to(BF).to(R.DEV), labels.to(R.DEV)
    assert torch.equal(w.cpu().float()[0, top, torch.arange(width)], tops)
    want = R.vocab_loss(h, w, None, labels)
    out = V.call(h, w, None, labels, F32, piece, only_loss=only_loss)
    assert torch.all((out[0].double() - want[0]).abs() <= 2.0 ** -22 + 4 * R.U * want[0])
    assert torch.all((out[1].double() - want[1]).abs() <= 2.0 ** -22 + 4 * R.U * want[1])
