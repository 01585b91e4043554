"""hdet_head_rotary and its backward pass against 64 bits: layouts, parts of heads, far positions, strides, in place, graphs; the stretched frequencies on the CPU."""
import math

import pytest
import torch

import heads_reference as R
import ops_reference as O
import paper_2604_24708_amd as H

gpu = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def inputs(n, rows, q_heads, k_heads, d, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(width, std=1.0):
        return (torch.randn(n, rows, width, generator=g, device=DEV) * std).to(dtype)

    q, k, dq, dk = normal(q_heads * d, 2.0), normal(k_heads * d, 0.5), normal(q_heads * d), normal(k_heads * d)
    gains = [1.0 + 0.2 * torch.randn(n, d, generator=g, device=DEV) for _ in range(2)]
    return q, k, dq, dk, gains


def bound(want, size, dtype, angle_err=0.0):
    """Rounding of the result, some fp32 operations on numbers of the pair's size, and the angle's error times it."""
    return R.half(dtype) * want.abs() + (24 * R.U + angle_err) * size


def pair_size(x, d):
    """The largest entry of the head."""
    return x.abs().view(*x.shape[:2], -1, d).amax(-1, keepdim=True).expand(*x.shape[:2], -1, d).reshape(x.shape)


def run_and_check(q, k, dq, dk, q_gain, k_gain, d, freq, pos=None, period=0, paired=False, magnitude=1.0, out=None, grads=None):
    n, rows, _ = dq.shape
    if pos is None:
        where = torch.arange(rows, device=DEV).expand(n, rows) % (period or rows + 1)
    else:
        where = pos
    how = dict(freq=freq, positions=pos, period=period, paired=paired, magnitude=magnitude, eps=EPS, q_gain=q_gain, k_gain=k_gain)
    q_out, k_out = out or [torch.full_like(x, 7.0) for x in (q, k)]
    H.hdet_head_rotary(q, q_out, d, k=k, k_out=k_out, **how)
    dq_in, dk_in = grads or [torch.full_like(x, 7.0) for x in (q, k)]
    gains = [None if g is None else torch.full((n, d), 7.0, device=DEV) for g in (q_gain, k_gain)]
    work = torch.full((H.hdet_head_rotary_backward_workspace(n, rows, d, q.shape[2] // d, k.shape[2] // d),), 0xff, dtype=torch.uint8, device=DEV)
    H.hdet_head_rotary_backward(q, dq, dq_in, d, k=k, dk_out=dk, dk=dk_in, dq_gain=gains[0], dk_gain=gains[1], workspace=work, **how)
    for name, x, y, dy, dx, gain, dgain in (("q", q, q_out, dq, dq_in, q_gain, gains[0]), ("k", k, k_out, dk, dk_in, k_gain, gains[1])):
        want = R.rotary(x, gain, d, where, freq, paired, magnitude, EPS)
        R.check(y, want, bound(want, (abs(magnitude) + 1) * pair_size(R.rotary(x, gain, d, where, None, paired, 1.0, EPS), d), x.dtype), name + "_out")
        wx, wg, size = R.rotary_backward(x, dy, gain, d, where, freq, paired, magnitude, EPS)
        # the mean's sum: terms of the size of w gain xh
        scale = (abs(magnitude) + 1) * pair_size(dy.double(), d)
        if gain is not None:
            u = x.double().view(n, rows, -1, d)
            rstd = (1.0 / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS))
            xh = (u * rstd).abs().amax(-1, keepdim=True)
            scale = scale * (rstd * (1.0 + xh * xh) * gain.double().abs().amax(-1).view(n, 1, 1, 1)).expand(u.shape).reshape(x.shape)
        R.check(dx, wx, bound(wx, scale, x.dtype), "d" + name)
        if gain is not None:
            # fp32 sums over rows and heads: in blocks and teams, chains of at most a few hundred additions; 24 roundings in a term
            heads = x.shape[2] // d
            longest = min(rows * heads, 700) + 24
            R.check(dgain, wg, R.U * longest * (size + pair_size(dy.double(), d).view(n, rows, -1, d).sum((1, 2)) * (abs(magnitude) + 1)), f"d{name}_gain")
    return q_out, k_out


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("paired", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("n,rows,q_heads,k_heads,d,rotated", [
    (1, 1, 1, 1, 1, 0), (2, 1, 2, 1, 2, 2), (1, 3, 5, 1, 7, 4), (2, 5, 4, 2, 16, 16), (1, 17, 8, 8, 64, 64), (3, 33, 6, 2, 64, 32), (2, 40, 3, 1, 80, 20),
    (1, 100, 16, 4, 128, 128), (2, 9, 2, 2, 128, 48), (1, 21, 2, 1, 256, 256), (1, 6, 3, 1, 250, 100), (2, 11, 5, 5, 96, 96), (1, 513, 12, 1, 72, 72), (1, 4, 2, 1, 255, 254),
    (1, 2100, 1, 1, 64, 64)])
def test_sizes(n, rows, q_heads, k_heads, d, rotated, paired, dtype):
    q, k, dq, dk, gains = inputs(n, rows, q_heads, k_heads, d, dtype, seed=rows + d)
    freq = R.frequencies(rotated) if rotated else None
    run_and_check(q, k, dq, dk, *gains, d, freq, paired=paired)
    run_and_check(q, k, dq, dk, None, None, d, freq, paired=paired, period=5, magnitude=1.25)
    run_and_check(q, k, dq, dk, gains[0], None, d, freq, paired=paired, period=2)


@gpu
@pytest.mark.parametrize("paired", [False, True], ids=["halves", "pairs"])
def test_far_positions(paired):
    """Any 32-bit position: in fp32 the angle of the fastest pair would be off by whole turns."""
    n, rows, d = 2, 64, 64
    q, k, dq, dk, gains = inputs(n, rows, 4, 2, d, F32, seed=1)
    pos = torch.randint(-2 ** 31, 2 ** 31, (n, rows), generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
    pos[0, :4] = torch.tensor([0, 2 ** 31 - 1, -2 ** 31, 1], dtype=torch.int32)
    run_and_check(q, k, dq, dk, *gains, d, R.frequencies(d), pos=pos, paired=paired)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-25, 1e-12, 1e18, 1e30])
def test_sizes_of_numbers(size, dtype):
    """Squares beyond fp32's range, in both directions: against the formula, where eps counts for all of it at the small end."""
    n, rows, d = 1, 8, 64
    q, k, _, _, gains = inputs(n, rows, 2, 1, d, dtype, seed=2)
    q, k = (q.double() * size).to(dtype), (k.double() * size).to(dtype)
    freq, pos = R.frequencies(d), torch.arange(rows, device=DEV).expand(n, rows)
    out = torch.empty_like(q), torch.empty_like(k)
    H.hdet_head_rotary(q, out[0], d, k=k, k_out=out[1], freq=freq, q_gain=gains[0], k_gain=gains[1], eps=EPS)
    for x, y, gain in ((q, out[0], gains[0]), (k, out[1], gains[1])):
        want = R.rotary(x, gain, d, pos, freq, False, 1.0, EPS)
        R.check(y, want, bound(want, 2 * pair_size(want, d) * 1.5, dtype), "out")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("row_pad,rep_pad,offset", [(8, 0, 0), (3, 5, 1), (64, 24, 8)])
@pytest.mark.parametrize("paired", [False, True], ids=["halves", "pairs"])
def test_strides_and_what_lies_between(paired, row_pad, rep_pad, offset, dtype):
    n, rows, d = 2, 30, 64
    q, k, dq, dk, gains = inputs(n, rows, 4, 2, d, dtype, seed=3)
    how = dict(row_pad=row_pad, rep_pad=rep_pad, offset=offset)
    sq, sk, sdq, sdk = (O.strided(x, **how) for x in (q, k, dq, dk))
    out, grads = [O.strided(torch.zeros_like(x), **how) for x in (q, k)], [O.strided(torch.zeros_like(x), **how) for x in (q, k)]
    run_and_check(sq, sk, sdq, sdk, *gains, d, R.frequencies(d), paired=paired, out=out, grads=grads)
    for x in out + grads:
        inside = torch.zeros_like(x._base, dtype=torch.bool)
        torch.as_strided(inside, x.shape, x.stride(), x.storage_offset()).fill_(True)
        assert bool(torch.isnan(x._base[~inside].float()).all())


@gpu
@pytest.mark.parametrize("d,rotated", [(64, 64), (50, 18)])
def test_in_place_and_alone(d, rotated):
    n, rows = 2, 40
    q, k, dq, dk, gains = inputs(n, rows, 4, 2, d, BF16, seed=4)
    freq = R.frequencies(rotated)
    q_out, k_out = run_and_check(q, k, dq, dk, *gains, d, freq)
    qk = torch.cat((q, k), -1)
    H.hdet_head_rotary(qk[..., :4 * d], qk[..., :4 * d], d, k=qk[..., 4 * d:], k_out=qk[..., 4 * d:], q_gain=gains[0], k_gain=gains[1], freq=freq, eps=EPS)
    assert torch.equal(qk[..., :4 * d], q_out) and torch.equal(qk[..., 4 * d:], k_out)
    alone = torch.empty_like(q)
    H.hdet_head_rotary(q, alone, d, q_gain=gains[0], freq=freq, eps=EPS)
    assert torch.equal(alone, q_out)
    # the gradient without a norm needs no inputs, and may take the place of what it comes from
    want, _, _ = R.rotary_backward(None, dq, None, d, torch.arange(rows, device=DEV).expand(n, rows), freq, False, 1.0, EPS)
    H.hdet_head_rotary_backward(None, dq, dq, d, freq=freq)
    R.check(dq, want, bound(want, 2 * pair_size(want, d) * 1.5, BF16), "dq")


@gpu
def test_no_rows():
    q = torch.empty(2, 0, 128, dtype=BF16, device=DEV)
    gain, dgain = torch.ones(2, 64, device=DEV), torch.full((2, 64), 7.0, device=DEV)
    H.hdet_head_rotary(q, q, 64, q_gain=gain, freq=R.frequencies(64))
    H.hdet_head_rotary_backward(q, q, q, 64, q_gain=gain, freq=R.frequencies(64), dq_gain=dgain)
    assert not dgain.any()


@gpu
def test_a_head_that_is_not_finite_stays_alone():
    n, rows, d = 1, 20, 64
    q, k, dq, dk, gains = inputs(n, rows, 4, 2, d, BF16, seed=5)
    clean = torch.empty_like(q)
    H.hdet_head_rotary(q, clean, d, q_gain=gains[0], freq=R.frequencies(d), eps=EPS)
    q[0, 7, 70] = float("nan")
    out = torch.empty_like(q)
    H.hdet_head_rotary(q, out, d, q_gain=gains[0], freq=R.frequencies(d), eps=EPS)
    assert bool(torch.isnan(out[0, 7, 64:128]).all())
    out[0, 7, 64:128] = clean[0, 7, 64:128]
    assert torch.equal(out, clean)


@gpu
def test_large_matrices():
    """More than 2^31 bytes in a replica."""
    n, rows, heads, d = 1, 2_000_001, 9, 64
    q = torch.randn(n, rows, heads * d, device=DEV, dtype=BF16, generator=torch.Generator(device=DEV).manual_seed(1))
    gain, freq = torch.ones(n, d, device=DEV), R.frequencies(d)
    out = torch.empty_like(q)
    H.hdet_head_rotary(q, out, d, q_gain=gain, freq=freq, eps=EPS)
    dgain, dq = torch.empty(n, d, device=DEV), torch.empty_like(q)
    work = torch.empty(H.hdet_head_rotary_backward_workspace(n, rows, d, heads), dtype=torch.uint8, device=DEV)
    H.hdet_head_rotary_backward(q, out, dq, d, q_gain=gain, freq=freq, eps=EPS, dq_gain=dgain, workspace=work)
    for part in (slice(0, 1000), slice(rows - 1000, rows)):
        pos = torch.arange(rows, device=DEV)[None, part]
        want = R.rotary(q[:, part], gain, d, pos, freq, False, 1.0, EPS)
        R.check(out[:, part], want, bound(want, 2 * pair_size(want, d) * 1.5, BF16), "out")
        back, _, _ = R.rotary_backward(q[:, part], out[:, part], gain, d, pos, freq, False, 1.0, EPS)
        # dy here is the rotated head itself, off by half a step: what is left of it after the mean is taken off is small
        R.check(dq[:, part], back, 2.0 ** -8 * back.abs() + 200 * R.U * pair_size(out[:, part].double(), d), "dq")


@gpu
def test_captured_and_replayed():
    n, rows, d = 2, 300, 64
    q, k, dq, dk, gains = inputs(n, rows, 4, 2, d, BF16, seed=6)
    freq = R.frequencies(d)
    pos = torch.arange(rows, dtype=torch.int32, device=DEV).repeat(n, 1)
    work = torch.zeros(H.hdet_head_rotary_backward_workspace(n, rows, d, 4, 2), dtype=torch.uint8, device=DEV)
    res = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k), torch.empty(n, d, device=DEV), torch.empty(n, d, device=DEV)]

    def step(to):
        s = torch.cuda.current_stream().cuda_stream
        how = dict(freq=freq, positions=pos, q_gain=gains[0], k_gain=gains[1], eps=EPS, stream=s)
        H.hdet_head_rotary(q, to[0], d, k=k, k_out=to[1], **how)
        H.hdet_head_rotary_backward(q, dq, to[2], d, k=k, dk_out=dk, dk=to[3], dq_gain=to[4], dk_gain=to[5], workspace=work, **how)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(res)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(res)
    for turn in range(3):
        q.normal_(generator=torch.Generator(device=DEV).manual_seed(turn))
        pos += 1000
        for x in res:
            x.fill_(float("nan"))
        g.replay()
        want = [torch.empty_like(x) for x in res]
        step(want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(res, want))


@gpu
def test_gradients_against_differences():
    n, rows, d = 1, 6, 12
    q, k, dq, dk, gains = inputs(n, rows, 2, 1, d, F32, seed=7)
    freq, pos = R.frequencies(8), torch.arange(rows, device=DEV).expand(n, rows)
    dx, dgain = torch.empty_like(q), torch.empty(n, d, device=DEV)
    work = torch.empty(H.hdet_head_rotary_backward_workspace(n, rows, d, 2), dtype=torch.uint8, device=DEV)
    H.hdet_head_rotary_backward(q, dq, dx, d, q_gain=gains[0], freq=freq, eps=EPS, magnitude=0.75, dq_gain=dgain, workspace=work)

    def value(x, gain):
        return float((R.rotary(x, gain, d, pos, freq, False, 0.75, EPS) * dq.double()).sum())

    for at in [(0, 0, 0), (0, 3, 5), (0, 5, 23), (0, 2, 13), (0, 1, 9)]:
        moved = [q.double().clone(), q.double().clone()]
        moved[0][at] += 1e-5
        moved[1][at] -= 1e-5
        # the step's square times a third derivative of some tens; fp32 roundings of the gradient
        assert abs((value(moved[0], gains[0]) - value(moved[1], gains[0])) / 2e-5 - float(dx[at])) <= 2e-5
    for c in range(d):
        moved = [gains[0].double().clone(), gains[0].double().clone()]
        moved[0][0, c] += 1e-5
        moved[1][0, c] -= 1e-5
        assert abs((value(q, moved[0]) - value(q, moved[1])) / 2e-5 - float(dgain[0, c])) <= 2e-5


# ---- frequencies (no GPU) -----------------------------------------------------------------------
def test_frequencies():
    d = 64
    plain = [10000.0 ** (-2.0 * t / d) for t in range(d // 2)]

    def freq(*a, **kw):
        return H.hdet_rotary_frequencies(*a, device="cpu", **kw).tolist()

    assert freq(d) == pytest.approx(plain, rel=1e-15)
    assert freq(0) == [] and freq(2) == [1.0]
    assert freq(d, factor=4.0) == pytest.approx([f / 4 for f in plain], rel=1e-15)
    base = freq(d, stretch=H.HDET_STRETCH_BASE, factor=8.0)
    assert base[0] == 1.0 and base[-1] == pytest.approx(plain[-1] / 8, rel=1e-12)
    assert all(a > b for a, b in zip(base, base[1:]))
    parts = freq(d, stretch=H.HDET_STRETCH_PARTS, factor=8.0, context=2048.0, slow=1.0, fast=32.0)
    for f, p in zip(parts, plain):
        turns = 2048 * p / (2 * math.pi)
        want = p if turns >= 32 else p / 8 if turns <= 1 else p * ((turns - 1) / 31 + (32 - turns) / 31 / 8)
        assert f == pytest.approx(want, rel=1e-13)
    for bad in [dict(rotated=3), dict(rotated=-2), dict(rotated=258), dict(rotated=8, base=0.0), dict(rotated=8, base=float("nan")), dict(rotated=8, factor=0.0),
                dict(rotated=8, stretch=3), dict(rotated=2, stretch=H.HDET_STRETCH_BASE, factor=2.0), dict(rotated=8, stretch=H.HDET_STRETCH_PARTS),
                dict(rotated=8, stretch=H.HDET_STRETCH_PARTS, context=10.0, slow=2.0, fast=2.0)]:
        with pytest.raises(H.HdetError) as e:
            H.hdet_rotary_frequencies(device="cpu", **bad)
        assert e.value.code == H.HDET_EINVAL
