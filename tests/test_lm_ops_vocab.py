"""The output layer with its loss in pieces of the vocabulary, against 64 bits."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def make(n, rows, width, classes, seed, spread=2.0, ignored=0.1):
    g = torch.Generator(device=R.DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=R.DEV)  # noqa: E731
    h = rnd(n, rows, width).to(BF)
    w = (rnd(n, classes, width) * spread * width ** -0.5).to(BF)
    bias = 0.3 * rnd(n, classes)
    labels = torch.randint(0, classes, (n, rows), generator=g, device=R.DEV, dtype=torch.int32)
    drop = torch.rand(n, rows, generator=g, device=R.DEV) < ignored
    labels[drop] = -100
    return h, w, bias, labels


def call(h, w, bias, labels, dw_dtype=F32, piece=0, only_loss=False):
    n, rows, width = h.shape
    classes = w.shape[1]
    nan = float("nan")
    loss, mean = torch.full((n, rows), nan, device=R.DEV), torch.full((n,), nan, device=R.DEV)
    work = torch.empty(H.hdet_vocab_loss_workspace(n, rows, width, classes, dw=dw_dtype, piece=piece), dtype=torch.uint8, device=R.DEV)
    work.fill_(0xff)                                       # nothing in it has to start at anything
    if only_loss:
        H.hdet_vocab_loss(h, w, labels, loss, mean, bias=bias, piece=piece, workspace=work)
        return loss, mean
    dh, dw = torch.full(h.shape, nan, dtype=BF, device=R.DEV), torch.full(w.shape, nan, dtype=dw_dtype, device=R.DEV)
    db = torch.full((n, classes), nan, device=R.DEV)
    H.hdet_vocab_loss(h, w, labels, loss, mean, dh=dh, dw=dw, bias=bias, db=db, piece=piece, workspace=work)
    return loss, mean, dh, dw, db


def check(out, h, w, bias, labels):
    """Logits are fp32 sums of exact products: off by (width + 2) U sum|h w|, L below.  What follows moves by as much in its logarithm, plus a few U of
    the exponents' arguments (below 64 U here).  Parts in bfloat16 are off by 2^-9 of themselves (2^-8 at most), and dh and a bfloat16 dw once more."""
    want = R.vocab_loss(h, w, bias, labels)
    loss, mean, dh, dw, db = out
    width = h.shape[2]
    L = (width + 2) * R.U * float(torch.matmul(h.double().abs(), w.double().abs().transpose(1, 2).contiguous()).max()) + 64 * R.U
    assert torch.all((loss.double() - want[0]).abs() <= 2 * L + 4 * R.U * want[0].abs())
    assert torch.all((mean.double() - want[1]).abs() <= 2 * L + 4 * R.U * want[1].abs())
    dz = want[5]
    c = ((labels >= 0) & (labels < w.shape[1])).sum(-1).clamp(min=1).double()[:, None, None]
    on = torch.zeros_like(dz).scatter_(-1, labels.long().clamp(0, w.shape[1] - 1)[..., None], 1.0) * (dz.abs().amax(-1, keepdim=True) > 0) / c
    p = (dz + on).abs()                                     # the softmax's share of dz
    rows, classes = h.shape[1], w.shape[1]
    size = dz.abs() + p                                     # in whose size dz is off
    assert torch.all((db.double() - want[4]).abs() <= (2 * L + (rows + 8) * R.U) * size.sum(1) + 1e-38)
    hw, hh = w.double().abs(), h.double().abs()
    sh, sw = torch.matmul(size, hw), torch.matmul(size.transpose(1, 2).contiguous(), hh)
    assert torch.all((dh.double() - want[2]).abs() <= (2.0 ** -8 + 2 * L + (classes + 2) * R.U) * sh + 2.0 ** -8 * want[2].abs() + 1e-38)
    rough = 2.0 ** -8 if dw.dtype == BF else 2.0 ** -23
    assert torch.all((dw.double() - want[3]).abs() <= (rough + 2 * L + (3 * rows + 2) * R.U) * sw + (2.0 ** -8 if dw.dtype == BF else R.U) * want[3].abs() + 1e-38)
    # over whole tensors: bfloat16 roundings of either kind are 2^-9 at most in the mean
    if float(want[2].norm()) > 0:
        assert R.rel(dh, want[2]) <= 2 * 2.0 ** -9
        # (dz as a difference of nearly equal numbers is less exact than its size says where a class is all but certain)
        assert R.rel(dw, want[3]) <= (2 * 2.0 ** -9 if dw.dtype == BF else 2e-6 + 4 * L)


SHAPES = [(1, 1, 1, 1, 0), (1, 1, 8, 3, 0), (2, 3, 5, 7, 0), (1, 2, 64, 100, 0), (3, 17, 40, 33, 0), (4, 128, 64, 512, 0), (2, 50, 72, 300, 64), (1, 129, 96, 1000, 256),
          (2, 200, 136, 777, 200), (1, 300, 256, 2048, 512), (2, 257, 200, 1504, 1000), (1, 64, 512, 4100, 1024), (1, 500, 100, 5003, 0), (2, 96, 1024, 640, 256),
          (1, 1000, 256, 1280, 0), (2, 512, 512, 2568, 768), (1, 40, 264, 9000, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,width,classes,piece", [s for s in SHAPES if s[4] != 1])
def test_loss_and_gradients(n, rows, width, classes, piece, dtype):
    h, w, bias, labels = make(n, rows, width, classes, classes)
    out = call(h, w, bias, labels, dtype, piece)
    check(out, h, w, bias, labels)
    again = call(h, w, bias, labels, dtype, piece)
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    loss, mean = call(h, w, bias, labels, dtype, piece, only_loss=True)
    ref = R.vocab_loss(h, w, bias, labels)
    L = (width + 2) * R.U * float(torch.matmul(h.double().abs(), w.double().abs().transpose(1, 2).contiguous()).max()) + 64 * R.U
    assert torch.all((loss.double() - ref[0]).abs() <= 2 * L + 4 * R.U * ref[0].abs())
    check(call(h, w, None, labels, dtype, piece), h, w, None, labels)


@pytest.mark.parametrize("width", [48, 256])
@pytest.mark.parametrize("piece", [0, 256, 300])
def test_rows_that_do_not_count(width, piece):
    n, rows, classes = 3, 70, 1032
    h, w, bias, labels = make(n, rows, width, classes, 1)
    labels[0] = -1                                          # a replica without any
    labels[1] = classes                                     # just past the last class
    labels[1, 5] = classes - 1
    labels[2, ::3] = 2 ** 31 - 1
    h[2, 0] = float("nan")                                  # of a row that does not count
    out = call(h, w, bias, labels, F32, piece)
    assert torch.all(out[0][0] == 0) and float(out[1][0]) == 0
    for t in out[2:]:
        assert torch.all(t[0] == 0)
    assert torch.all(out[2][1, :5] == 0) and torch.all(out[2][1, 6:] == 0) and bool((out[2][1, 5] != 0).any())
    assert torch.all(out[0][2, ::3] == 0) and torch.all(torch.isfinite(out[0]))
    assert torch.all(torch.isfinite(out[4]))
    h[2, 0] = 0
    out = call(h, w, bias, labels, F32, piece)
    check(out, h, w, bias, labels)


@pytest.mark.parametrize("width", [40, 256])
@pytest.mark.parametrize("piece", [0, 256])
def test_masked_classes(width, piece):
    """A bias of -inf takes classes out, whole pieces among them; a row whose label is masked is infinite, others are not touched by it."""
    n, rows, classes = 1, 60, 1024
    h, w, bias, labels = make(n, rows, width, classes, 2, ignored=0.0)
    bias[0, :600] = -float("inf")
    labels.copy_(600 + labels % (classes - 600))
    out = call(h, w, bias, labels, F32, piece)
    keep = slice(600, None)
    few = call(h, w[:, keep].contiguous(), bias[:, keep].contiguous(), (labels - 600).contiguous(), F32, 0)
    ref = R.vocab_loss(h, w[:, keep], bias[:, keep], labels - 600)
    assert torch.all((out[0].double() - ref[0]).abs() <= 1e-5 * (1 + ref[0].abs()))
    assert torch.all(out[3][:, :600] == 0) and torch.all(out[4][:, :600] == 0)
    assert R.rel(out[3][:, keep], ref[3]) <= 1e-5 and R.rel(out[2], ref[2]) <= 2 * 2.0 ** -9
    assert torch.all((few[0] - out[0]).abs() <= 1e-5 * (1 + out[0].abs()))
    labels[0, 3] = 5
    out = call(h, w, bias, labels, F32, piece)
    assert torch.isinf(out[0][0, 3]) and torch.all(torch.isfinite(out[0][0, 4:]))


@pytest.mark.parametrize("width", [40, 256])
@pytest.mark.parametrize("size", [30.0, 300.0])
def test_large_logits(width, size):
    """Logits of a few hundred: the reference keeps exponentials in range, and rows differ by as much."""
    n, rows, classes = 1, 64, 1024
    h, w, bias, labels = make(n, rows, width, classes, 3, spread=size)
    check(call(h, w, bias, labels, F32, 256), h, w, bias, labels)


def test_strides():
    """Operands inside larger matrices, gradients inside parameter planes of any alignment."""
    n, rows, width, classes = 2, 150, 264, 1000
    h, w, bias, labels = make(n, rows, width, classes, 4)
    want = call(h, w, bias, labels, F32, 0)
    for dtype in (BF, F32):
        for pad, rep, off in [(8, 64, 8), (1, 3, 1), (4, 4, 4)]:
            hs, ws = R.strided(h, pad, rep, off), R.strided(w, pad, rep, off)
            dh = R.strided(torch.zeros_like(h), pad, rep, off)
            dw = R.strided(torch.zeros(n, classes, width, dtype=dtype, device=R.DEV), pad, rep, off)
            db = torch.full((n, classes + 9), float("nan"), device=R.DEV)
            loss, mean = torch.empty(n, rows, device=R.DEV), torch.empty(n, device=R.DEV)
            for piece in (0, 256):
                work = torch.empty(H.hdet_vocab_loss_workspace(n, rows, width, classes, dw=dtype, piece=piece), dtype=torch.uint8, device=R.DEV)
                H.hdet_vocab_loss(hs, ws, labels, loss, mean, dh=dh, dw=dw, bias=bias, db=db[:, 3:3 + classes], piece=piece, workspace=work)
                check((loss, mean, dh, dw, db[:, 3:3 + classes]), h, w, bias, labels)
            assert torch.all(torch.isnan(db[:, :3])) and torch.all(torch.isnan(db[:, 3 + classes:]))
            gaps = torch.as_strided(dw, (n, classes, width + pad), dw.stride(), dw.storage_offset())[:, : classes - 1, width:]
            assert torch.all(torch.isnan(gaps))
    assert torch.isfinite(want[1]).all()


def test_no_rows():
    n, width, classes = 2, 40, 33
    h, w = torch.empty(n, 0, width, dtype=BF, device=R.DEV), torch.zeros(n, classes, width, dtype=BF, device=R.DEV)
    labels = torch.empty(n, 0, dtype=torch.int32, device=R.DEV)
    out = call(h, w, None, labels, F32, 0)
    assert torch.all(out[1] == 0) and torch.all(out[3] == 0) and torch.all(out[4] == 0)


@pytest.mark.parametrize("width,classes", [(48, 300), (256, 1024)])
def test_gradient_against_differences(width, classes):
    """Differences of the mean loss between neighbouring bfloat16 inputs and between biases: second-order terms cancel in central differences, third-order
    ones are at most step^3; the mean loss itself is exact to 8 U of its size (logits to L)."""
    n, rows = 1, 40
    h, w, bias, labels = make(n, rows, width, classes, 6)
    loss, mean, dh, dw, db = call(h, w, bias, labels, F32, 256)
    L = (width + 2) * R.U * float(torch.matmul(h.double().abs(), w.double().abs().transpose(1, 2).contiguous()).max()) / 8 + 8 * R.U * float(mean)
    g = torch.Generator(device=R.DEV).manual_seed(3)
    for which in ("h", "w", "bias"):
        t, grad = {"h": (h, dh), "w": (w, dw), "bias": (bias, db)}[which]
        v = grad.double() / grad.double().abs().max()       # along the gradient, where the change is largest
        v = v + 0.1 * torch.randn(t.shape, generator=g, device=R.DEV) * v.abs().mean()
        up, down = (t.double() + 0.05 * v).to(t.dtype), (t.double() - 0.05 * v).to(t.dtype)
        args = {"h": lambda x: (x, w, bias), "w": lambda x: (h, x, bias), "bias": lambda x: (h, w, x)}[which]
        a = call(*args(up), labels, F32, 256, only_loss=True)[1]
        b = call(*args(down), labels, F32, 256, only_loss=True)[1]
        step = up.double() - down.double()
        want = float((grad.double() * step).sum())
        got = float(a.double() - b.double())
        assert abs(want) > 20 * L
        assert abs(got - want) <= 4 * L + 0.02 * abs(want)
