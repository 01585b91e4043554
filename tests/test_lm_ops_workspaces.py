"""Scratch memory of the language-model operators: what a call asks for is what it uses, and no more than it needs for the results it is given."""
import ctypes as C
import math
import random
import re

import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H
from paper_2604_24708_amd import binding as B

P = 1 << 40            # an aligned address that nothing reads
BF, F32 = torch.bfloat16, torch.float32


def asked_for(name, args):
    """The workspace that a call says it needs, given one byte too few of it: refused before anything is enqueued."""
    args.workspace_dev, args.workspace_bytes = P, 0
    assert getattr(H.load_library(), name)(C.byref(args), None) == H.HDET_EINVAL
    return int(re.search(r"(\d+) bytes are needed", H.hdet_last_error()).group(1))


def vocab_args(n, rows, width, classes, piece, dw_dtype, dh=True, dw=True, db=True):
    m = lambda r: B.hdet_rows(P, width, r * width)  # noqa: E731
    a = B.hdet_vocab_args(n_replicas=n, dw_dtype=dw_dtype, rows=rows, width=width, classes=classes, piece=piece, labels_dev=P, row_loss_dev=P, mean_loss_dev=P, h=m(rows), w=m(classes))
    if dh:
        a.dh = m(rows)
    if dw:
        a.dw = m(classes)
    if db:
        a.db_dev, a.db_stride = P, classes
    return a


def vocab_sizes():
    rng = random.Random(5)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    drawn = [(rng.choice([1, 2, 3, 4, 5, 8, 64]), log(1, 30000), log(1, 4096), log(1, 200000), rng.choice([0, 0, 0, 5, 300, 4096])) for _ in range(1500)]
    return [(8, 4096, 512, 32000, 0), (4, 8192, 1024, 32000, 0), (8, 521, 64, 105157, 0)] + drawn


def test_a_loss_without_dw_needs_no_more_than_with_one():
    for n, rows, width, classes, piece in vocab_sizes():
        s = lambda dh, dw, db, t=H.HDET_TYPE_F32: asked_for("hdet_vocab_loss", vocab_args(n, rows, width, classes, piece, t, dh, dw, db))  # noqa: E731
        full = [s(True, True, True, t) for t in (H.HDET_TYPE_F32, H.HDET_TYPE_BF16)]
        size = lambda dw: H.hdet_vocab_loss_workspace(n, rows, width, classes, dw=dw, piece=piece)  # noqa: E731
        assert full == [size(F32), size(BF)] and size(None) == size(F32)
        for t in (H.HDET_TYPE_F32, H.HDET_TYPE_BF16):
            some, none = s(True, False, True, t), s(False, False, False, t)
            assert none <= some <= min(full), (n, rows, width, classes, piece, none, some, full)
            assert s(True, False, False, t) == s(False, False, True, t) == some
            assert some == size(H.HDET_VOCAB_NO_DW) and none == size(H.HDET_VOCAB_LOSSES)


def test_the_losses_alone_need_no_gradient_of_the_logits():
    """8 x 4096 rows of 512, 32000 classes: 1 GB in a call with gradients; without, a reference and a sum for each row and 256 classes, or 128 MB of logits."""
    assert H.hdet_vocab_loss_workspace(8, 4096, 512, 32000, dw=H.HDET_VOCAB_LOSSES) < 144 << 20
    for bad in (-3, 2):
        with pytest.raises(H.HdetError):
            H.hdet_vocab_loss_workspace(1, 1, 1, 1, dw=bad)


def test_the_size_for_a_dw_that_the_call_would_refuse_is_refused():
    with pytest.raises(ValueError):
        H.hdet_vocab_loss_workspace(1, 1, 1, 1, dw=torch.float16)


def guarded(size):
    """`size` bytes of scratch memory, and what lies behind them."""
    t = torch.full((size + 4096,), 0xa5, dtype=torch.uint8, device=R.DEV)
    return t[:size], t[size:]


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows,width,classes,piece", [(2, 50, 72, 300, 64), (1, 100, 96, 9600, 0), (2, 300, 333, 8200, 2048), (1, 1900, 264, 2304, 0), (8, 521, 64, 105157, 0)])
def test_a_loss_stays_inside_its_workspace(n, rows, width, classes, piece):
    import test_lm_ops_vocab as V
    h, w, bias, labels = V.make(n, rows, width, classes, 12)
    nan = float("nan")
    want = None
    for dw_dtype, dw in ((F32, True), (BF, True), (H.HDET_VOCAB_NO_DW, False), (H.HDET_VOCAB_LOSSES, False)):
        work, behind = guarded(H.hdet_vocab_loss_workspace(n, rows, width, classes, dw=dw_dtype, piece=piece))
        grads = dict(dh=torch.full_like(h, nan), db=torch.full((n, classes), nan, device=R.DEV)) if dw_dtype != H.HDET_VOCAB_LOSSES else {}
        if dw:
            grads["dw"] = torch.full(w.shape, nan, dtype=dw_dtype, device=R.DEV)
        loss, mean = torch.full((n, rows), nan, device=R.DEV), torch.full((n,), nan, device=R.DEV)
        H.hdet_vocab_loss(h, w, labels, loss, mean, bias=bias, piece=piece, workspace=work, **grads)
        assert torch.all(behind == 0xa5)
        out = (loss, mean, *(grads[k] for k in ("dh", "db") if k in grads))
        if want is None:
            want = out
            for z in range(n):
                ref = R.vocab_loss(h[z:z + 1], w[z:z + 1], bias[z:z + 1], labels[z:z + 1])
                assert torch.all((loss[z:z + 1].double() - ref[0]).abs() <= 1e-5 * (1 + ref[0].abs())) and R.rel(grads["dh"][z:z + 1], ref[2]) <= 2 * 2.0 ** -9
                assert R.rel(grads["dw"][z:z + 1], ref[3]) <= 1e-5 and R.rel(grads["db"][z:z + 1], ref[4]) <= 1e-5
                del ref
        # pieces differ between the calls, and with them the order of fp32 sums
        assert torch.all((loss - want[0]).abs() <= 1e-5 * (1 + want[0].abs())) and torch.all((mean - want[1]).abs() <= 1e-5 * (1 + want[1].abs()))
        if grads:
            assert R.rel(grads["dh"], want[2].double()) <= 2 * 2.0 ** -9 and R.rel(grads["db"], want[3].double()) <= 1e-5


def test_no_rows_need_no_workspace_for_a_loss():
    for dw in (F32, BF, H.HDET_VOCAB_NO_DW, H.HDET_VOCAB_LOSSES):
        assert H.hdet_vocab_loss_workspace(3, 0, 777, 50000, dw=dw) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dw_dtype", [BF, F32])
@pytest.mark.parametrize("width,classes", [(8, 300), (333, 9000)])
def test_a_loss_without_rows(width, classes, dw_dtype):
    n = 3
    h, w = torch.empty(n, 0, width, dtype=BF, device=R.DEV), torch.ones(n, classes, width, dtype=BF, device=R.DEV)
    labels, loss = torch.empty(n, 0, dtype=torch.int32, device=R.DEV), torch.empty(n, 0, device=R.DEV)
    mean, db = torch.full((n,), 7.0, device=R.DEV), torch.full((n, classes + 5), 7.0, device=R.DEV)
    dw = R.strided(torch.zeros(n, classes, width, device=R.DEV).to(dw_dtype), 3, 2, 1).fill_(7)
    H.hdet_vocab_loss(h, w, labels, loss, mean, dh=torch.empty_like(h), dw=dw, db=db[:, 2:2 + classes])
    assert torch.all(mean == 0) and torch.all(dw == 0) and torch.all(db[:, 2:2 + classes] == 0) and torch.all(db[:, :2] == 7) and torch.all(db[:, 2 + classes:] == 7)
    mean.fill_(7)
    H.hdet_vocab_loss(h, w, labels, loss, mean)
    assert torch.all(mean == 0)


def linear_grad_args(n, rows, d_in, d_out, dx=True, dw=True, db=True):
    wide = -(-d_in // 16) * 16
    a = B.hdet_linear_grad_args(n_replicas=n, rows=rows, d_in=d_in, d_out=d_out, scale_dev=P, w_scale_dev=P, dy=B.hdet_rows(P, d_out, rows * d_out),
                                codes=B.hdet_rows(P, wide, rows * wide), w_codes=B.hdet_rows(P, wide, d_out * wide))
    if dx:
        a.dx = B.hdet_rows(P, d_in, rows * d_in)
    if dw:
        a.dw = B.hdet_rows(P, d_in, d_out * d_in)
    if db:
        a.db_dev, a.db_stride = P, d_out
    return a


def test_linear_gradients_ask_for_what_their_results_need():
    """bfloat16 copies of W for dx and of X for dw; neither for db."""
    for n, rows, d_in, d_out in [(8, 8192, 1024, 4096), (3, 5150, 776, 1501), (1, 20000, 64, 40), (2, 1000, 9000, 24)]:
        s = lambda *on: asked_for("hdet_quantised_linear_backward", linear_grad_args(n, rows, d_in, d_out, *on))  # noqa: E731
        full, dx, dw, db = s(True, True, True), s(True, False, False), s(False, True, False), s(False, False, True)
        assert full == H.hdet_quantised_linear_backward_workspace(n, rows, d_in, d_out) and max(dx, dw, db) <= full
        pitch, ragged = -(-d_in // 8) * 8, d_out % 8 != 0
        more = n * rows * (d_out + 8) * 2 if ragged else 0             # dy in whole pieces
        parts = 256 * 128 * 128 * 4 * 2                                # results of pieces of a contraction: half the compute units' tiles at most, each in up to twice as many
        assert n * d_out * pitch * 2 <= dx <= n * d_out * pitch * 2 + more + parts
        assert n * rows * pitch * 2 <= dw <= n * rows * pitch * 2 + more + parts
        assert db <= n * (rows // 16 + 1) * d_out * 4 + 256
        assert full <= n * (rows + d_out) * pitch * 2 + more + parts + db + 1024
    assert H.hdet_quantised_linear_backward_workspace(3, 0, 777, 50000) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows,d_in,d_out", [(3, 129, 300, 131), (2, 257, 384, 1024), (1, 2000, 96, 72), (2, 130, 264, 1664), (1, 9, 40, 33)])
def test_linear_gradients_stay_inside_their_workspace(n, rows, d_in, d_out):
    import test_lm_ops_linear as L
    x, xs, w, ws, _, dy = L.make(n, rows, d_in, d_out, 13)
    new = lambda: dict(dx=torch.empty(n, rows, d_in, dtype=BF, device=R.DEV), dw=torch.empty(n, d_out, d_in, device=R.DEV), db=torch.empty(n, d_out, device=R.DEV))  # noqa: E731
    want = None
    for on in (("dx", "dw", "db"), ("dx",), ("dw",), ("db",), ("dw", "db"), ("dx", "db")):
        out = {k: v for k, v in new().items() if k in on}
        size = 0
        if on != ("db",) or rows > 16:
            size = asked_for("hdet_quantised_linear_backward", linear_grad_args(n, rows, d_in, d_out, *(k in on for k in ("dx", "dw", "db"))))
        work, behind = guarded(size)
        H.hdet_quantised_linear_backward(dy, x, xs, w, ws, workspace=work if size else None, **out)
        assert torch.all(behind == 0xa5)
        if want is None:
            want = out
            d = dy.double()
            assert R.rel(out["dx"], torch.matmul(d, L.values(w, ws))) <= R.half_ulp(BF)
            assert R.rel(out["dw"], torch.matmul(d.transpose(1, 2).contiguous(), L.values(x, xs))) <= 8 * R.U * rows ** 0.5
            assert torch.all((out["db"].double() - d.sum(1)).abs() <= (rows + 2) * R.U * d.abs().sum(1))
        assert all(torch.equal(out[k], want[k]) for k in on)


@pytest.mark.gpu
def test_linear_gradients_without_rows_need_no_workspace():
    n, d_in, d_out = 2, 72, 40
    x, w = H.hdet_codes_empty(n, 0, d_in), H.hdet_codes_empty(n, d_out, d_in)
    db, dw = torch.ones(n, d_out, device=R.DEV), torch.ones(n, d_out, d_in, device=R.DEV)
    dy, dx = torch.empty(n, 0, d_out, dtype=BF, device=R.DEV), torch.empty(n, 0, d_in, dtype=BF, device=R.DEV)
    H.hdet_quantised_linear_backward(dy, x, torch.empty(n, 0, device=R.DEV), w, torch.ones(n, d_out, device=R.DEV), dx=dx, dw=dw, db=db)
    assert torch.all(db == 0) and torch.all(dw == 0)


def test_scratch_in_host_memory_is_refused():
    with pytest.raises(ValueError, match="workspace is on cpu"):
        B._work_of(torch.empty(1 << 20, dtype=torch.uint8))
    assert B._work_of(None) == (None, 0)


@pytest.mark.gpu
def test_scratch_with_gaps_is_refused():
    """The library takes a pointer and a number of bytes: every other byte of a buffer, or one of them many times, is no such memory.  Nothing is enqueued."""
    n, rows, width = 2, 40, 64
    x, gain, rstd = torch.ones(n, rows, width, device=R.DEV), torch.ones(n, width, device=R.DEV), torch.ones(n, rows, device=R.DEV)
    size = H.hdet_rmsnorm_backward_workspace(n, rows, width)
    buf = torch.full((2 * size,), 0x5a, dtype=torch.uint8, device=R.DEV)
    h, labels = torch.ones(n, rows, width, dtype=BF, device=R.DEV), torch.zeros(n, rows, dtype=torch.int32, device=R.DEV)
    codes, w = H.hdet_codes_empty(n, rows, width), H.hdet_codes_empty(n, 24, width)
    for work in (buf[::2], buf[:1].expand(1 << 30)):
        for call in (lambda: H.hdet_rmsnorm_backward(x, gain, rstd, x, torch.empty_like(x), dgain=torch.empty_like(gain), workspace=work),
                     lambda: H.hdet_vocab_loss(h, h, labels, rstd, torch.empty(n, device=R.DEV), workspace=work),
                     lambda: H.hdet_quantised_linear_backward(h[..., :24], codes, rstd, w, torch.ones(n, 24, device=R.DEV), dx=torch.empty_like(h), workspace=work)):
            with pytest.raises(ValueError, match="workspace must be contiguous"):
                call()
    torch.cuda.synchronize()
    assert torch.all(buf == 0x5a)
