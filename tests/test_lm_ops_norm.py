"""Root-mean-square norm with residual and 8-bit output, its backward pass, rows to 8 bits and back, against 64 bits."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
EPS = 1e-5
BF, F32 = torch.bfloat16, torch.float32


def make(n, rows, width, dtype, seed):
    g = torch.Generator(device=R.DEV).manual_seed(seed)
    x = (torch.randn(n, rows, width, generator=g, device=R.DEV) * torch.exp(torch.randn(n, rows, 1, generator=g, device=R.DEV))).to(dtype)
    r = torch.randn(n, rows, width, generator=g, device=R.DEV).to(dtype)
    gain = 1.0 + 0.3 * torch.randn(n, width, generator=g, device=R.DEV)
    dy = torch.randn(n, rows, width, generator=g, device=R.DEV).to(dtype)
    dt = torch.randn(n, rows, width, generator=g, device=R.DEV).to(dtype)
    return x, r, gain, dy, dt


# the longest chain of additions over a row: 32 in a thread, 6 across a wavefront, 16 across a block; the square root halves it, 4 more roundings
def rstd_bound():
    return (54 / 2 + 4) * R.U


def check_codes(codes, scale, y, width):
    """codes and scale are those of y up to the error of the kernel's own fp32 y."""
    err = rstd_bound() + 3 * R.U
    s = scale.double()
    top = y.abs().amax(-1)
    assert torch.all(torch.frexp(scale)[0] == 0.5)
    assert torch.all(127 * s >= top * (1 - err))
    assert torch.all((127 * s / 2 < top * (1 + err)) | (scale == 2.0 ** -126))
    v = codes.double() * s[..., None]
    assert torch.all((v - y).abs() <= s[..., None] / 2 * (1 + 1e-12) + err * y.abs())
    assert int(codes.abs().max()) <= 127
    padded = torch.as_strided(codes, (*codes.shape[:2], (width + 15) // 16 * 16), codes.stride(), codes.storage_offset())
    assert torch.all(padded[..., width:] == 0)


def check_forward(x, r, gain, total, y, codes, scale, rstd):
    u, rs, yy = R.norm(x, r, gain, EPS)
    hu = R.half_ulp(x.dtype)
    assert torch.all((total.double() - u).abs() <= (hu + R.U) * u.abs())
    assert torch.all((rstd.double() - rs).abs() <= rstd_bound() * rs)
    assert torch.all((y.double() - yy).abs() <= (hu + rstd_bound() + 3 * R.U) * yy.abs() + 1e-38)
    check_codes(codes, scale, yy, x.shape[-1])


def check_backward(total, gain, rstd, dy, dt, dx, dgain):
    want, wg = R.norm_backward(total, gain, rstd, dy, dt)
    h, r, g, d = total.double(), rstd.double()[..., None], gain.double()[:, None], dy.double()
    size = r * ((d * g).abs() + (h * r).abs() * (d * g * h * r).abs().mean(-1, keepdim=True)) + (0 if dt is None else dt.double().abs())
    assert torch.all((dx.double() - want).abs() <= R.half_ulp(dx.dtype) * want.abs() + (54 + 8) * R.U * size)
    if dgain is not None:
        rows = h.shape[1]
        assert torch.all((dgain.double() - wg).abs() <= (rows + 8) * R.U * (d * h * r).abs().sum(1) + 1e-38)
        assert R.rel(dgain, wg) <= 8 * R.U * max(1.0, rows ** 0.5)


SHAPES = [(1, 1, 1), (2, 3, 7), (1, 5, 8), (3, 33, 64), (2, 17, 72), (1, 9, 120), (2, 65, 136), (1, 3, 255), (2, 30, 256), (8, 40, 512), (2, 7, 513), (1, 300, 520),
          (2, 19, 1000), (3, 5, 1024), (1, 6, 1032), (1, 4, 2047), (2, 11, 2048), (1, 3, 2056), (1, 5, 4096), (1, 2, 5001), (2, 3, 8192), (1, 2, 8200), (1, 3, 16384),
          (1, 2, 20000), (1, 2, 32761), (1, 1, 32768), (1, 4099, 96), (2, 2500, 264)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,width", SHAPES)
def test_forward_and_backward(n, rows, width, dtype):
    x, r, gain, dy, dt = make(n, rows, width, dtype, width * 7 + rows)
    total, y, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    codes, scale, rstd = H.hdet_codes_empty(n, rows, width), torch.empty(n, rows, device=R.DEV), torch.empty(n, rows, device=R.DEV)
    torch.as_strided(codes, (n, rows, codes.stride(1)), codes.stride()).fill_(99)          # the padding is written, not left
    H.hdet_rmsnorm(x, gain, resid=r, total=total, y=y, codes=codes, scale=scale, rstd=rstd, eps=EPS)
    check_forward(x, r, gain, total, y, codes, scale, rstd)
    values = torch.empty(n, rows, width, dtype=BF, device=R.DEV)
    H.hdet_restore_rows(codes, scale, values)
    assert torch.equal(values.double(), codes.double() * scale.double()[..., None])         # a bfloat16 number, exactly
    dgain = torch.empty(n, width, device=R.DEV)
    work = torch.empty(max(16, H.hdet_rmsnorm_backward_workspace(n, rows, width)), dtype=torch.uint8, device=R.DEV)
    H.hdet_rmsnorm_backward(total, gain, rstd, dy, dx, dtotal=dt, dgain=dgain, workspace=work)
    check_backward(total, gain, rstd, dy, dt, dx, dgain)
    again, dgain2 = torch.empty_like(dx), torch.empty_like(dgain)
    H.hdet_rmsnorm_backward(total, gain, rstd, dy, again, dtotal=dt, dgain=dgain2, workspace=work)
    assert torch.equal(again, dx) and torch.equal(dgain, dgain2)                            # fixed orders: the same bits


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("row_pad,rep_pad,offset", [(8, 0, 0), (24, 40, 16), (1, 0, 0), (0, 3, 5), (3, 1, 2)])
def test_strides_absent_operands_and_in_place(dtype, row_pad, rep_pad, offset):
    n, rows, width = 3, 21, 136
    x, r, gain, dy, dt = make(n, rows, width, dtype, 5)
    pad = lambda t: R.strided(t, row_pad, rep_pad, offset)  # noqa: E731
    xs, rs = pad(x), pad(r)
    y = pad(torch.zeros_like(x))
    H.hdet_rmsnorm(xs, gain, resid=rs, y=y, eps=EPS)
    want = torch.empty_like(x)
    H.hdet_rmsnorm(x, gain, resid=r, y=want, eps=EPS)
    u, rstd64, yy = R.norm(x, r, gain, EPS)
    assert torch.all((y.double() - yy).abs() <= (R.half_ulp(dtype) + rstd_bound() + 3 * R.U) * yy.abs())
    assert torch.all((want.double() - yy).abs() <= (R.half_ulp(dtype) + rstd_bound() + 3 * R.U) * yy.abs())
    # without a residual, only the codes
    codes, scale = H.hdet_codes_empty(n, rows, width), torch.empty(n, rows, device=R.DEV)
    H.hdet_rmsnorm(xs, gain, codes=codes, scale=scale, eps=EPS)
    check_codes(codes, scale, R.norm(x, None, gain, EPS)[2], width)
    # the sum over its own summand, the gradient over the incoming one, one gain for all replicas
    gain1 = gain[:1].expand(n, width)
    rstd, total, dx = torch.empty(n, rows, device=R.DEV), pad(x), pad(dt)
    H.hdet_rmsnorm(total, gain1, resid=rs, total=total, rstd=rstd, eps=EPS)
    assert torch.all((total.double() - u).abs() <= (R.half_ulp(dtype) + R.U) * u.abs())
    H.hdet_rmsnorm_backward(total, gain1, rstd, pad(dy), dx, dtotal=dx)
    check_backward(total, gain1, rstd, dy, dt, dx, None)
    # nothing between the rows has been written
    buf = torch.as_strided(dx, (n, rows, width + row_pad), dx.stride(), dx.storage_offset())
    assert torch.all(torch.isnan(buf[..., width:]))


def test_one_gradient_for_all_rows_and_no_rows():
    n, width = 2, 48
    gain = torch.ones(n, width, device=R.DEV)
    x = torch.empty(n, 0, width, device=R.DEV)
    dgain = torch.full((n, width), 5.0, device=R.DEV)
    H.hdet_rmsnorm(x, gain, y=torch.empty_like(x))
    H.hdet_rmsnorm_backward(x, gain, torch.empty(n, 0, device=R.DEV), x, torch.empty_like(x), dgain=dgain)
    assert torch.all(dgain == 0)
    # a broadcast incoming gradient (row stride 0)
    x, r, gain, dy, dt = make(2, 50, 64, F32, 3)
    rstd, dx = torch.empty(2, 50, device=R.DEV), torch.empty_like(x)
    H.hdet_rmsnorm(x, gain, rstd=rstd, eps=EPS)
    # replicas may share their input: stride 0 between them
    shared = x[:1].expand_as(x)
    y1, y2 = torch.empty_like(x), torch.empty_like(x)
    H.hdet_rmsnorm(shared, gain, y=y1, eps=EPS)
    H.hdet_rmsnorm(shared.contiguous(), gain, y=y2, eps=EPS)
    assert torch.equal(y1, y2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("width", [37, 64, 1024, 4000])
def test_special_rows(dtype, width):
    """Rows of zeros, of the type's extremes, and with entries that are not finite."""
    big = torch.finfo(dtype).max
    x = torch.zeros(1, 9, width, device=R.DEV)
    x[0, 1] = 1e-30
    x[0, 2, 3] = 1.0
    x[0, 3] = 3.0
    x[0, 4, 5] = float("inf")
    x[0, 5, 6] = float("nan")
    x[0, 6, 7] = -float("inf")
    x[0, 7] = torch.linspace(-127, 127, width, device=R.DEV)
    x[0, 8, 0], x[0, 8, 1] = big, -big
    x = x.to(dtype)
    codes, scale = H.hdet_codes_empty(1, 9, width), torch.empty(1, 9, device=R.DEV)
    H.hdet_quantise_rows(x, codes, scale)
    fine = [0, 1, 2, 3, 7, 8]
    want, ws = R.rows8(x[:, fine].double())
    assert torch.equal(scale[:, fine].double(), ws[..., 0])
    assert torch.equal(codes[:, fine].double(), want)                   # a power of two: the codes are exact
    assert torch.all(torch.isnan(scale[:, 4:7])) and torch.all(codes[:, 4:7] == 0)
    values = torch.empty(1, 9, width, dtype=dtype, device=R.DEV)
    H.hdet_restore_rows(codes, scale, values)
    assert torch.all(torch.isnan(values[:, 4:7])) and torch.all(torch.isfinite(values[:, fine[:-1]]))
    # the type's largest number is 63.75 (63.99..) steps of 2^122 and reads back as 64 of them, which is 2^128
    assert float(values[0, 8, 0]) == float("inf") and float(values[0, 8, 2]) == 0
    # the norm: rows of zeros stay zeros, rows that are not finite are marked
    gain = torch.ones(1, width, device=R.DEV)
    H.hdet_rmsnorm(x, gain, codes=codes, scale=scale, eps=EPS)
    assert torch.all(codes[0, 0] == 0) and float(scale[0, 0]) == 2.0 ** -126
    assert torch.all(torch.isnan(scale[:, 4:7])) and torch.all(codes[:, 4:7] == 0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,rows,width", [(1, 1, 1), (2, 7, 33), (3, 100, 512), (1, 3, 10000), (2, 5, 2048)])
def test_rows_to_8_bits_exactly(n, rows, width, dtype):
    x = make(n, rows, width, dtype, width)[0]
    x[0, 0, 0] = 127.0                     # the very edge of a scale
    codes, scale = H.hdet_codes_empty(n, rows, width), torch.empty(n, rows, device=R.DEV)
    H.hdet_quantise_rows(x, codes, scale)
    want, s = R.rows8(x.double())
    assert torch.equal(codes.double(), want) and torch.equal(scale.double(), s[..., 0])
    wide = torch.empty(n, rows, 20, device=R.DEV)                      # values into a matrix of other strides and type
    if width == 33:
        out = R.strided(torch.zeros(n, rows, width, device=R.DEV), 5, 2, 3)
        H.hdet_restore_rows(codes, scale, out)
        assert torch.equal(out.double(), want * s)
    del wide


def test_gradient_against_differences():
    """Central differences of L = sum(dy y) + sum(dt total) in fp32 along random directions: off by the third derivative times step^2 / 6 and by the
    roundings of y, at most U * sum|dy y| * 40 / step."""
    n, rows, width = 2, 4, 96
    x, r, gain, dy, dt = make(n, rows, width, F32, 11)

    def value(x, gain):
        y, t, rs = torch.empty_like(x), torch.empty_like(x), torch.empty(n, rows, device=R.DEV)
        H.hdet_rmsnorm(x, gain, resid=r, total=t, y=y, rstd=rs, eps=EPS)
        return float((dy.double() * y.double()).sum() + (dt.double() * t.double()).sum()), t, rs, float((dy.double() * y.double()).abs().sum())

    _, total, rstd, size = value(x, gain)
    dx, dgain = torch.empty_like(x), torch.empty_like(gain)
    work = torch.empty(H.hdet_rmsnorm_backward_workspace(n, rows, width), dtype=torch.uint8, device=R.DEV)
    H.hdet_rmsnorm_backward(total, gain, rstd, dy, dx, dtotal=dt, dgain=dgain, workspace=work)
    g = torch.Generator(device=R.DEV).manual_seed(2)
    step = 2.0 ** -7
    for _ in range(4):
        v = torch.randn(x.shape, generator=g, device=R.DEV)
        up, down = x + step * v, x - step * v
        got = (value(up, gain)[0] - value(down, gain)[0]) / 2
        want = float((dx.double() * (up.double() - down.double()) / 2).sum())
        # third derivatives of u / |u| are of the size of 10 / rms^2 times the entry, rms >= 1 here
        assert abs(got - want) <= size * (40 * R.U + 10 * step ** 3)
        v = torch.randn(gain.shape, generator=g, device=R.DEV)
        up, down = gain + step * v, gain - step * v
        got = (value(x, up)[0] - value(x, down)[0]) / 2
        want = float((dgain.double() * (up.double() - down.double()) / 2).sum())
        assert abs(got - want) <= size * 40 * R.U          # linear in the gain


def test_on_another_stream():
    x, r, gain, _, _ = make(4, 500, 512, BF, 1)
    want, got = torch.empty_like(x), torch.empty_like(x)
    H.hdet_rmsnorm(x, gain, resid=r, y=want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x2 = x + 0
        H.hdet_rmsnorm(x2, gain, resid=r, y=got, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(want, got)
