"""Matrices of more than 2^31 bytes, and more than 2^32 elements, in one replica: whole calls against calls on their last rows, or against 64 bits."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H
import test_lm_ops_vocab as V

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def random_rows(rows, width, dtype, seed):
    """A matrix [1, rows, width] of which no two rows are alike, quickly: shifts of one long random row, each times a number of its own."""
    g = torch.Generator(device=R.DEV).manual_seed(seed)
    x = torch.empty(1, rows, width, dtype=dtype, device=R.DEV)
    line = torch.randn(width + 997, generator=g, device=R.DEV)
    size = torch.exp(torch.randn(rows, generator=g, device=R.DEV))
    for a in range(0, rows, 4096):
        n = min(4096, rows - a)
        shift = (torch.arange(a, a + n, device=R.DEV) % 997)[:, None]
        x[0, a:a + n] = (line[shift + torch.arange(width, device=R.DEV)] * size[a:a + n, None]).to(dtype)
    return x


@pytest.mark.parametrize("rows,width", [(140001, 32768), (530001, 8200)])
def test_norm_and_8_bit_rows(rows, width):
    """More than 2^32 entries: the last rows are those of a call on them alone, bit for bit."""
    assert rows * width > 1 << 32
    x = random_rows(rows, width, BF, 1)
    gain = 1.0 + 0.1 * torch.randn(1, width, device=R.DEV, generator=torch.Generator(device=R.DEV).manual_seed(2))
    new = lambda x: (torch.empty_like(x), H.hdet_codes_empty(*x.shape), torch.empty(x.shape[:2], device=R.DEV), torch.empty(x.shape[:2], device=R.DEV))  # noqa: E731
    y, codes, scale, rstd = new(x)
    H.hdet_rmsnorm(x, gain, y=y, codes=codes, scale=scale, rstd=rstd)
    tail = x[:, -600:].contiguous()
    y2, codes2, scale2, rstd2 = new(tail)
    H.hdet_rmsnorm(tail, gain, y=y2, codes=codes2, scale=scale2, rstd=rstd2)
    assert torch.equal(y[:, -600:], y2) and torch.equal(codes[:, -600:], codes2) and torch.equal(scale[:, -600:], scale2) and torch.equal(rstd[:, -600:], rstd2)
    dx, dx2 = torch.empty_like(x), torch.empty_like(tail)
    H.hdet_rmsnorm_backward(x, gain, rstd, y, dx, dtotal=y)
    H.hdet_rmsnorm_backward(tail, gain, rstd2, y2, dx2, dtotal=y2)
    assert torch.equal(dx[:, -600:], dx2)
    H.hdet_quantise_rows(x, codes, scale)
    H.hdet_quantise_rows(tail, codes2, scale2)
    assert torch.equal(codes[:, -600:], codes2) and torch.equal(scale[:, -600:], scale2)
    H.hdet_restore_rows(codes, scale, dx)
    H.hdet_restore_rows(codes2, scale2, dx2)
    assert torch.equal(dx[:, -600:], dx2)
    del x, y, dx, codes
    torch.cuda.empty_cache()


def codes_of(rows, width, seed):
    g = torch.Generator(device=R.DEV).manual_seed(seed)
    c = H.hdet_codes_empty(1, rows, width)
    for a in range(0, rows, 8192):
        c[:, a:a + 8192] = torch.randint(-127, 128, c[:, a:a + 8192].shape, generator=g, device=R.DEV, dtype=torch.int8)
    return c, torch.exp2(torch.randint(-8, 8, (1, rows), generator=g, device=R.DEV).float())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", [(17001, 131056, 4104), (17001, 131056, 49), (1100000, 33, 2056), (1100001, 33, 2001)])
def test_quantised_linear(rows, d_in, d_out, dtype):
    """Codes of more than 2^31 bytes, or results of more than 2^31 elements.  Sums of code products are exact: every kernel gives the same bits."""
    x, xs = codes_of(rows, d_in, 3)
    w, ws = codes_of(d_out, d_in, 4)
    y = torch.empty(1, rows, d_out, dtype=dtype, device=R.DEV)
    H.hdet_quantised_linear(x, xs, w, ws, y)
    for part in (slice(0, 40), slice(rows - 40, rows), slice(rows - 7, rows)):
        few = torch.empty(1, part.stop - part.start, d_out, dtype=dtype, device=R.DEV)
        H.hdet_quantised_linear(x[:, part].contiguous() if d_in % 16 == 0 else x[:, part], xs[:, part].contiguous(), w, ws, few)
        assert torch.equal(y[:, part], few)
    del x, y
    torch.cuda.empty_cache()


def test_gradients_of_the_linear_layer():
    """X in bfloat16 takes 2.2 GB: more than the kernels with 32-bit offsets take."""
    rows, d_in, d_out = 140000, 8000, 400
    x, xs = codes_of(rows, d_in, 5)
    w, ws = codes_of(d_out, d_in, 6)
    dy = random_rows(rows, d_out, BF, 7)
    dx, dw, db = torch.empty(1, rows, d_in, dtype=BF, device=R.DEV), torch.empty(1, d_out, d_in, device=R.DEV), torch.empty(1, d_out, device=R.DEV)
    work = torch.empty(H.hdet_quantised_linear_backward_workspace(1, rows, d_in, d_out), dtype=torch.uint8, device=R.DEV)
    H.hdet_quantised_linear_backward(dy, x, xs, w, ws, dx=dx, dw=dw, db=db, workspace=work)
    vw = w[0].double() * ws[0].double()[:, None]
    want_w, size_w = torch.zeros(d_out, d_in, dtype=torch.float64, device=R.DEV), torch.zeros(d_out, d_in, dtype=torch.float64, device=R.DEV)
    want_b = torch.zeros(d_out, dtype=torch.float64, device=R.DEV)
    for a in range(0, rows, 20000):
        d, v = dy[0, a:a + 20000].double(), x[0, a:a + 20000].double() * xs[0, a:a + 20000].double()[:, None]
        want_x = torch.matmul(d, vw)
        assert torch.all((dx[0, a:a + 20000].double() - want_x).abs() <= R.half_ulp(BF) * want_x.abs() + (d_out + 2) * R.U * torch.matmul(d.abs(), vw.abs()))
        want_w += torch.matmul(d.t().contiguous(), v)
        size_w += torch.matmul(d.abs().t().contiguous(), v.abs())
        want_b += d.sum(0)
    assert torch.all((dw[0].double() - want_w).abs() <= (rows + 2) * R.U * size_w)
    assert R.rel(dw[0], want_w) <= 8 * R.U * rows ** 0.5 and R.rel(db[0], want_b) <= 8 * R.U * rows ** 0.5
    del x, dx, dy, work
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,width,classes,piece,pad", [(20003, 64, 60008, 60008, 0), (4100, 72, 400003, 0, 0), (20003, 64, 60008, 30000, 1)])
def test_loss(rows, width, classes, piece, pad, dtype):
    """A gradient of the logits of 2.4 GB, or of 7.2 in three parts, in one piece; 400000 classes; logits through memory.  Bounds on whole tensors as in test_lm_ops_vocab."""
    h, w, bias, labels = V.make(1, rows, width, classes, 1)
    hs, ws = (R.strided(h, 1, 0, 1), R.strided(w, 1, 0, 1)) if pad else (h, w)
    loss, mean, dh, dw, db = V.call(hs, ws, bias, labels, dtype, piece)
    ok = ((labels >= 0) & (labels < classes))[0]
    c = float(ok.sum())
    want_w = torch.zeros(classes, width, dtype=torch.float64, device=R.DEV)
    want_b, want_loss = torch.zeros(classes, dtype=torch.float64, device=R.DEV), torch.zeros(rows, dtype=torch.float64, device=R.DEV)
    want_h = torch.zeros(rows, width, dtype=torch.float64, device=R.DEV)
    w64 = w[0].double()
    for a in range(0, rows, 1024):
        part = slice(a, min(a + 1024, rows))
        z = torch.matmul(h[0, part].double(), w64.t().contiguous()) + bias[0].double()
        at = labels[0, part].long().clamp(0, classes - 1)[:, None]
        lse = torch.logsumexp(z, -1, keepdim=True)
        want_loss[part] = torch.where(ok[part], (lse - z.gather(1, at))[:, 0], torch.zeros_like(want_loss[part]))
        p = torch.exp(z - lse)
        p.scatter_add_(1, at, torch.full_like(lse, -1.0))
        p *= ok[part].double()[:, None] / c
        want_h[part] = torch.matmul(p, w64)
        want_w += torch.matmul(p.t().contiguous(), h[0, part].double())
        want_b += p.sum(0)
    L = (width + 2) * R.U * float((h[0, :2048].double().abs() @ w64.abs().t().contiguous()).max()) * 2 + 64 * R.U
    assert torch.all((loss[0].double() - want_loss).abs() <= 2 * L + 4 * R.U * want_loss.abs())
    assert abs(float(mean) - float(want_loss.sum()) / c) <= 2 * L + 4 * R.U * float(want_loss.sum()) / c
    assert R.rel(dh[0], want_h) <= 2 * 2.0 ** -9
    assert R.rel(dw[0], want_w) <= (2 * 2.0 ** -9 if dtype == BF else 2e-6 + 4 * L)
    assert R.rel(db[0], want_b) <= 2e-6 + 4 * L
    # the last rows by themselves, against the last rows of dh
    assert R.rel(dh[0, -500:], want_h[-500:]) <= 2 * 2.0 ** -9 and R.rel(dw[0, -500:], want_w[-500:]) <= (2 * 2.0 ** -8 if dtype == BF else 1e-5 + 4 * L)
    del dw, w64
    torch.cuda.empty_cache()
