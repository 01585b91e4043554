"""The norm's 8-bit output is the formula's, code for code: sums, norm and rounding to codes hold more than fp32."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [1000, 1024])
def test_codes_are_the_formulas(width, dtype):
    """In 64 bits the kernel's y and the one here differ by a few 2^-53 times the length of a sum of squares, 2^-40 of themselves at most: a code can only differ where y / scale lies that near
    to a half.  The scale is taken from the row's largest entry in fp32: rows within 2^-23 of the edge between two scales are left out, and (bfloat16) those whose sum x + resid is no
    fp32 number.  In 32 bits y is off by up to 3e-7 of itself and about one row of 800 has a code one off: 40 of these rows."""
    n, rows = 2, 16384
    g = torch.Generator(device=R.DEV).manual_seed(width)
    x = torch.randn(n, rows, width, generator=g, device=R.DEV).to(dtype)
    r = torch.randn(n, rows, width, generator=g, device=R.DEV).to(dtype)
    gain = 1.0 + 0.1 * torch.randn(n, width, generator=g, device=R.DEV)
    codes, scale = H.hdet_codes_empty(n, rows, width), torch.empty(n, rows, device=R.DEV)
    H.hdet_rmsnorm(x, gain, resid=r, codes=codes, scale=scale, eps=1e-5)
    used = 0
    for z in range(n):
        u, _, y = R.norm(x[z:z + 1], r[z:z + 1], gain[z:z + 1], 1e-5)
        q, s = R.rows8(y)
        top = y.abs().amax(-1)
        edge = torch.minimum((top / (127.0 * s[..., 0]) - 1).abs(), (2 * top / (127.0 * s[..., 0]) - 1).abs())
        ok = edge > 2.0 ** -23
        if dtype == torch.bfloat16:
            ok &= ((x[z:z + 1].float() + r[z:z + 1].float()).double() == u).all(-1)
        assert torch.equal(scale[z:z + 1][ok].double(), s[..., 0][ok])
        v = y / s
        near = ((v - torch.floor(v)) - 0.5).abs() <= v.abs() * 2.0 ** -40
        assert torch.all((codes[z:z + 1].double() == q) | near | ~ok[..., None])
        used += int(ok.sum())
    assert used > 0.9 * n * rows
