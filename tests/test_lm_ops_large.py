"""The language-model operators at sizes that take their kernels for large calls: blocks that walk over several tiles, rows past the caches, long contractions of unaligned rows."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H
import test_lm_ops_linear as L
import test_lm_ops_norm as N
import test_lm_ops_vocab as V

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
PAST_CACHES = 256 << 20        # bytes of a launch from which on rows go past the caches


def tiles(n, rows, cols):
    return n * -(-rows // 256) * -(-cols // 256)


# more tiles of 256 x 256 than the 256 compute units, ragged at both edges: K of one chunk, of a step and a half, of several steps, and of an odd number of them
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,d_in,d_out", [(8, 1030, 200, 1800), (8, 1300, 7, 1544), (4, 2600, 520, 2056), (1, 4100, 1290, 8200), (3, 5001, 640, 1320)])
def test_quantised_linear_walks_over_tiles(n, rows, d_in, d_out, dtype):
    assert tiles(n, rows, d_out) > 256
    L.test_forward(n, rows, d_in, d_out, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantised_linear_walks_inside_larger_matrices(dtype):
    """Results in rows and replicas further apart, at 16-byte boundaries; nothing between them is written; rows without a scale stay alone."""
    n, rows, d_in, d_out = 5, 2100, 100, 1616
    x, xs, w, ws, bias, _ = L.make(n, rows, d_in, d_out, 2)
    y = R.strided(torch.zeros(n, rows, d_out, dtype=dtype, device=R.DEV), 24, 40, 16)
    assert tiles(n, rows, d_out) > 256
    H.hdet_quantised_linear(x, xs, w, ws, y, bias=bias)
    L.check_y(y, x, xs, w, ws, bias)
    gaps = torch.as_strided(y, (n, rows, d_out + 24), y.stride(), y.storage_offset())[:, : rows - 1, d_out:]
    assert torch.all(torch.isnan(gaps))
    xs[2, 1000] = float("nan")
    H.hdet_quantised_linear(x, xs, w, ws, y, bias=bias)
    bad = torch.isnan(y).any(-1)
    assert bool(torch.isnan(y[2, 1000]).all()) and int(bad.sum()) == 1


# several tiles a block in both passes, dz in one and in three parts; whole and in pieces of more than a round
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,width,classes,piece", [(2, 1100, 72, 8300, 0), (1, 2100, 200, 17001, 0), (3, 1030, 264, 10003, 8192), (8, 600, 520, 4099, 0)])
def test_loss_walks_over_tiles(n, rows, width, classes, piece, dtype):
    assert tiles(n, rows, min(classes, piece or classes)) > 256
    V.test_loss_and_gradients(n, rows, width, classes, piece, dtype)


def reference_in_parts(f, rows, *ts):
    """f over slices of the rows, each in 64 bits."""
    for a in range(0, rows, 2048):
        f(*(t[:, a:a + 2048] for t in ts))


@pytest.mark.parametrize("dtype,n,rows,width", [(BF, 2, 8200, 2056), (F32, 2, 8200, 1032), (BF, 3, 45000, 256), (F32, 1, 4200, 4096)])
def test_norm_past_the_caches(dtype, n, rows, width):
    assert 4 * (2 if dtype == BF else 4) * n * rows * width > PAST_CACHES          # (the backward pass, and the sum with y; codes add to it)
    x, r, gain, dy, dt = N.make(n, rows, width, dtype, 3)
    total, y, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    codes, scale, rstd = H.hdet_codes_empty(n, rows, width), torch.empty(n, rows, device=R.DEV), torch.empty(n, rows, device=R.DEV)
    H.hdet_rmsnorm(x, gain, resid=r, total=total, y=y, codes=codes, scale=scale, rstd=rstd, eps=N.EPS)
    dgain = torch.empty(n, width, device=R.DEV)
    work = torch.empty(H.hdet_rmsnorm_backward_workspace(n, rows, width), dtype=torch.uint8, device=R.DEV)
    H.hdet_rmsnorm_backward(total, gain, rstd, dy, dx, dtotal=dt, dgain=dgain, workspace=work)
    want, size = torch.zeros(n, width, dtype=torch.float64, device=R.DEV), torch.zeros(n, width, dtype=torch.float64, device=R.DEV)

    def part(x, r, total, y, codes, scale, rstd, dy, dt, dx):
        N.check_forward(x, r, gain, total, y, codes, scale, rstd)
        N.check_backward(total, gain, rstd, dy, dt, dx, None)
        xh = dy.double() * total.double() * rstd.double()[..., None]
        want.add_(xh.sum(1))
        size.add_(xh.abs().sum(1))
    reference_in_parts(part, rows, x, r, total, y, codes, scale, rstd, dy, dt, dx)
    assert torch.all((dgain.double() - want).abs() <= (rows + 8) * R.U * size + 1e-38)
    assert R.rel(dgain, want) <= 8 * R.U * rows ** 0.5
    # the gradient over the incoming one, and the sum over its summand
    H.hdet_rmsnorm_backward(total, gain, rstd, dy, dt, dtotal=dt)
    assert torch.equal(dt, dx)
    H.hdet_rmsnorm(x, gain, resid=r, total=x, y=dx, eps=N.EPS)
    assert torch.equal(x, total) and torch.equal(dx, y)


@pytest.mark.parametrize("dtype,n,rows,width", [(BF, 1, 88000, 1024), (F32, 2, 26600, 1024)])
def test_rows_to_8_bits_past_the_caches(dtype, n, rows, width):
    assert (3 if dtype == BF else 5) * n * rows * width > PAST_CACHES
    x = N.make(n, rows, width, dtype, 4)[0]
    codes, scale = H.hdet_codes_empty(n, rows, width), torch.empty(n, rows, device=R.DEV)
    H.hdet_quantise_rows(x, codes, scale)

    def part(x, codes, scale):
        want, s = R.rows8(x.double())
        assert torch.equal(codes.double(), want) and torch.equal(scale.double(), s[..., 0])
    reference_in_parts(part, rows, x, codes, scale)


def test_row_sums_past_the_caches():
    n, rows, d_in, d_out = 2, 16400, 16, 4104
    assert 2 * n * rows * d_out > PAST_CACHES
    g = torch.Generator(device=R.DEV).manual_seed(1)
    dy = torch.randn(n, rows, d_out, generator=g, device=R.DEV).to(BF)
    x, w = H.hdet_codes_empty(n, rows, d_in), H.hdet_codes_empty(n, d_out, d_in)
    db = torch.full((n, d_out), float("nan"), device=R.DEV)
    work = torch.empty(H.hdet_quantised_linear_backward_workspace(n, rows, d_in, d_out), dtype=torch.uint8, device=R.DEV)
    H.hdet_quantised_linear_backward(dy, x, torch.zeros(n, rows, device=R.DEV), w, torch.zeros(n, d_out, device=R.DEV), db=db, workspace=work)
    want, size = torch.zeros_like(db, dtype=torch.float64), torch.zeros_like(db, dtype=torch.float64)

    def part(d):
        want.add_(d.double().sum(1))
        size.add_(d.double().abs().sum(1))
    reference_in_parts(part, rows, dy)
    assert torch.all((db.double() - want).abs() <= (rows + 2) * R.U * size)
    assert R.rel(db, want) <= 8 * R.U * rows ** 0.5


@pytest.mark.parametrize("row_pad,rep_pad,offset", [(1, 3, 1), (2, 0, 0), (4, 4, 4)])
@pytest.mark.parametrize("n,rows,d_in,d_out", [(1, 2000, 96, 72), (2, 130, 264, 1664), (1, 1700, 40, 1608)])
def test_long_contractions_of_unaligned_rows(n, rows, d_in, d_out, row_pad, rep_pad, offset):
    """Few tiles and 1536 or more of the contraction, where dy's rows start at any element."""
    x, xs, w, ws, _, dy = L.make(n, rows, d_in, d_out, 5)
    dys = R.strided(dy, row_pad, rep_pad, offset)
    dx = R.strided(torch.zeros(n, rows, d_in, dtype=BF, device=R.DEV), row_pad, rep_pad, offset)
    dw = R.strided(torch.zeros(n, d_out, d_in, device=R.DEV), row_pad, rep_pad, offset)
    db = torch.empty(n, d_out, device=R.DEV)
    work = torch.empty(H.hdet_quantised_linear_backward_workspace(n, rows, d_in, d_out), dtype=torch.uint8, device=R.DEV)
    H.hdet_quantised_linear_backward(dys, x, xs, w, ws, dx=dx, dw=dw, db=db, workspace=work)
    vx, vw, d = L.values(x, xs), L.values(w, ws), dy.double()
    want_x, want_w = torch.matmul(d, vw), torch.matmul(d.transpose(1, 2).contiguous(), vx)
    size_x, size_w = torch.matmul(d.abs(), vw.abs()), torch.matmul(d.abs().transpose(1, 2).contiguous(), vx.abs())
    assert torch.all((dx.double() - want_x).abs() <= R.half_ulp(BF) * want_x.abs() + (d_out + 2) * R.U * size_x)
    assert torch.all((dw.double() - want_w).abs() <= (rows + 2) * R.U * size_w)
    assert R.rel(dw, want_w) <= 8 * R.U * rows ** 0.5
    assert torch.all((db.double() - d.sum(1)).abs() <= (rows + 2) * R.U * d.abs().sum(1))
    for t, c in ((dx, d_in), (dw, d_out)):
        cols = t.shape[2]
        gaps = torch.as_strided(t, (n, t.shape[1], cols + row_pad), t.stride(), t.storage_offset())[:, : t.shape[1] - 1, cols:]
        assert torch.all(torch.isnan(gaps))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,width,classes", [(100, 96, 9600), (1800, 64, 700)])
def test_loss_of_unaligned_rows_with_a_long_contraction(rows, width, classes, dtype):
    h, w, bias, labels = V.make(1, rows, width, classes, 7)
    out = V.call(R.strided(h, 1, 0, 1), R.strided(w, 1, 0, 1), bias, labels, dtype, 0)
    V.check(out, h, w, bias, labels)
