"""hdet_clip_gradients against 64 bits: tensors of all kinds and many of them, in place and into a plane, shared gradients, norms at the ends of the range, graphs."""
import math

import pytest
import torch

import heads_reference as R
import ops_reference as O
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def make(n, shapes, seed=0, std=1.0, types=(F32,)):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(n, *s, generator=g, device=DEV) * std).to(types[i % len(types)]) for i, s in enumerate(shapes)]


def norms(grads, n, shared):
    if shared:
        total = sum(g.double().mean(0).square().sum() for g in grads) if grads else torch.zeros((), dtype=torch.float64, device=DEV)
        return torch.sqrt(total).expand(n)
    return torch.sqrt(sum(g.double().reshape(n, -1).square().sum(1) for g in grads))


def clip(grads, max_norm, outs=None, shared=False, n=None, stream=None, places=None):
    n = grads[0].shape[0] if n is None else n
    norm = torch.full((n,), 7.0, device=DEV)
    work = torch.full((H.hdet_clip_gradients_workspace(n, len(grads)),), 0xff, dtype=torch.uint8, device=DEV)
    H.hdet_clip_gradients(places or H.hdet_gradient_list(grads, outs), norm, max_norm, shared=shared, workspace=work, stream=stream)
    return norm


def check(grads, max_norm, shared=False, outs=None):
    n = grads[0].shape[0]
    want = norms(grads, n, shared)
    before = [g.clone() for g in grads]
    norm = clip(grads, max_norm, outs, shared)
    # 64-bit sums, rounded to fp32
    R.check(norm, want, 2 * R.U * want, "norm")
    factor = torch.where((want > max_norm) & torch.isfinite(want), max_norm / want, torch.ones_like(want))
    for i, (g, b) in enumerate(zip(grads, before)):
        x = b.double() * factor.view(n, *([1] * (b.dim() - 1)))
        if outs is None:
            # the factor's rounding and the product's, then the type's
            R.check(g, x, (4 * R.U + (R.half(g.dtype) if g.dtype == BF16 else 0)) * x.abs() + 2.0 ** -133, f"gradient {i}")
        else:
            assert torch.equal(g, b)
            R.check(outs[i], x, 4 * R.U * x.abs() + 2.0 ** -149, f"out {i}")
    return norm, factor


SHAPES = [(1,), (3,), (64,), (7, 5), (33, 64), (1, 8191), (8192,), (8193,), (100, 333), (257, 1024)]


@pytest.mark.parametrize("shared", [False, True], ids=["own", "shared"])
@pytest.mark.parametrize("n", [1, 2, 5, 64])
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F32, BF16)], ids=["f32", "bf16", "both"])
def test_kinds(types, n, shared):
    grads = make(n, SHAPES, seed=n, types=types)
    size = float(norms(grads, n, shared).min())
    _, factor = check(grads, size * 0.5, shared)
    assert bool((factor < 1).all())
    grads = make(n, SHAPES, seed=n, types=types)
    kept = [g.clone() for g in grads]
    check(grads, float(norms(grads, n, shared).max()) * 1.5, shared)
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))       # not a bit of them moves below the bound


@pytest.mark.parametrize("shared", [False, True], ids=["own", "shared"])
@pytest.mark.parametrize("step", [4, 1], ids=["aligned", "anywhere"])
def test_into_a_plane(step, shared):
    n = 3
    grads = make(n, SHAPES, seed=1, types=(F32, BF16))
    places, at = [], 0
    for s in SHAPES:
        places.append(at)
        at += -(-math.prod(s) // step) * step + (0 if step == 4 else 3)
    plane = torch.full((n, at + 5), float("nan"), device=DEV)
    outs = [plane[:, p:p + math.prod(s)].unflatten(1, s) for p, s in zip(places, SHAPES)]
    for max_norm in (float(norms(grads, n, shared).mean()) * 0.9, math.inf, 0.0):
        plane.fill_(float("nan"))
        check(grads, max_norm, shared, outs)
        inside = torch.zeros_like(plane, dtype=torch.bool)
        for p, s in zip(places, SHAPES):
            inside[:, p:p + math.prod(s)] = True
        assert bool(torch.isnan(plane[~inside]).all()) and bool(torch.isfinite(plane[inside]).all())


@pytest.mark.parametrize("count", [0, 1, 39, 40, 41, 300])
def test_numbers_of_tensors(count):
    n = 2
    grads = make(n, [((i * 37) % 500 + 1,) if i % 3 else ((i % 7) + 1, (i * 11) % 90 + 1) for i in range(count)], seed=2, types=(F32, F32, BF16))
    if not count:
        norm = clip([], 1.0, n=n)
        assert not norm.any()
        return
    check(grads, 3.0)
    outs = [torch.empty(g.shape, device=DEV) for g in grads]
    check(make(n, [g.shape[1:] for g in grads], seed=3), 2.0, outs=outs)


def test_empty_tensors():
    grads = [torch.empty(2, 0, device=DEV), torch.full((2, 3), 2.0, device=DEV), torch.empty(2, 0, 5, device=DEV), torch.empty(2, 4, 0, device=DEV)]
    norm = clip(grads, 1.0)
    assert norm.tolist() == pytest.approx([12.0 ** 0.5] * 2, rel=1e-6)
    assert grads[1].flatten().tolist() == pytest.approx([12.0 ** -0.5 * 2] * 6, rel=1e-6)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("row_pad,rep_pad,offset", [(8, 0, 0), (3, 5, 1), (64, 24, 8), (0, 7, 3)])
def test_strides_and_what_lies_between(row_pad, rep_pad, offset, dtype):
    n = 2
    for rows, width in ((40, 64), (300, 72), (9, 1001)):
        g = make(n, [(rows, width)], seed=4, types=(dtype,))[0]
        s = O.strided(g, row_pad=row_pad, rep_pad=rep_pad, offset=offset)
        check([s], 5.0)
        inside = torch.zeros_like(s._base, dtype=torch.bool)
        torch.as_strided(inside, s.shape, s.stride(), s.storage_offset()).fill_(True)
        assert bool(torch.isnan(s._base[~inside].float()).all())
        out = O.strided(torch.zeros(n, rows, width, device=DEV), row_pad=row_pad, rep_pad=rep_pad, offset=offset)
        check([O.strided(g, row_pad=5, rep_pad=1, offset=3)], 5.0, outs=[out])


def test_ends_of_the_range():
    """Squares beyond fp32, in both directions."""
    for std in (1e-30, 1e25):
        grads = make(2, [(1000,), (50, 60)], std=std)
        check(grads, std)
        check(make(2, [(1000,)], std=std), math.inf)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_norm_that_is_not_finite(bad):
    grads = make(2, [(1000,), (50, 60)], seed=5)
    grads[1][1, 3, 4] = bad
    kept = [g.clone() for g in grads]
    norm = clip(grads, 1.0)
    assert not math.isfinite(float(norm[1]))
    # that replica's gradients are left as they are; the other's are bounded
    assert all(torch.equal(a[1].nan_to_num(7.0), b[1].nan_to_num(7.0)) for a, b in zip(grads, kept))
    want = norms([g[:1] for g in kept], 1, False)
    R.check(grads[0][:1], kept[0][:1].double() / want, 4 * R.U * kept[0][:1].double().abs() / want, "gradient")


def test_shared_gradients_that_cancel():
    """The mean's norm, not the mean of norms."""
    g = make(1, [(3000,)], seed=6)[0]
    grads = [torch.cat((g, -g, g, -g))]
    norm = clip(grads, 1e-3, shared=True)
    assert not norm.any() and torch.equal(grads[0][0], g[0])


def test_large_tensors():
    """More than 2^32 bytes in a replica, and more than 2^31 elements."""
    n = 1
    big = torch.full((n, 2 ** 16, 2 ** 15 + 8), 0.5, dtype=BF16, device=DEV)
    assert big[0].numel() > 2 ** 31
    tail = big[:, -1, -5:].clone()
    norm = clip([big], 1.0)
    want = 0.5 * math.sqrt(big[0].numel())
    assert float(norm[0]) == pytest.approx(want, rel=2e-7)
    assert bool((big == torch.tensor(0.5 / want).to(BF16).to(DEV)).all()) and tail.numel() == 5


def test_captured_and_replayed():
    n = 3
    for count in (5, 60):
        grads = make(n, [(17 + i, 33) for i in range(count)], seed=7)
        outs = [torch.empty_like(g) for g in grads]
        places = H.hdet_gradient_list(grads, outs)
        norm, work = torch.empty(n, device=DEV), torch.zeros(H.hdet_clip_gradients_workspace(n, count), dtype=torch.uint8, device=DEV)

        def step():
            H.hdet_clip_gradients(places, norm, 2.0, workspace=work, stream=torch.cuda.current_stream().cuda_stream)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for turn in range(3):
            for x in grads:
                x.normal_(generator=torch.Generator(device=DEV).manual_seed(turn))
            norm.fill_(float("nan"))
            for x in outs:
                x.fill_(float("nan"))
            g.replay()
            got = [norm.clone(), *(x.clone() for x in outs)]
            step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, [norm, *outs]))


def test_the_same_bits_every_time():
    grads = make(4, SHAPES * 8, seed=8)
    first = clip(grads, math.inf)
    for _ in range(3):
        assert torch.equal(clip(grads, math.inf), first)
