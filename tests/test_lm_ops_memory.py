"""The language-model operators on memory beyond 32-bit offsets, inside captured graphs and on streams of their own."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FAR = (1 << 32) + 64          # elements between two replicas


def far(t, fill):
    """t [2, rows, cols] with FAR elements between the replicas."""
    buf = torch.empty(FAR + t.shape[1] * t.stride(1) + 64, dtype=t.dtype, device=R.DEV)
    v = torch.as_strided(buf, t.shape, (FAR, t.stride(1), 1))
    v.copy_(t) if fill else v.zero_()
    return v


def test_replicas_further_apart_than_32_bits():
    g = torch.Generator(device=R.DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device=R.DEV)  # noqa: E731
    rows, width = 70, 264
    x, gain = rnd(2, rows, width).to(BF), 1 + 0.1 * rnd(2, width)
    y, yf = torch.empty_like(x), None
    H.hdet_rmsnorm(x, gain, y=y)
    xf = far(x, True)
    yf = far(torch.empty_like(x), False)
    H.hdet_rmsnorm(xf, gain, y=yf)
    assert torch.equal(yf, y)
    del xf, yf
    codes, scale = H.hdet_codes_empty(2, rows, width), torch.empty(2, rows, device=R.DEV)
    H.hdet_quantise_rows(x, codes, scale)
    cf, sf = far(codes, False), torch.empty_like(scale)
    H.hdet_quantise_rows(x, cf, sf)
    assert torch.equal(cf, codes) and torch.equal(sf, scale)
    d_out = 520
    w, ws = H.hdet_codes_empty(2, d_out, width), torch.empty(2, d_out, device=R.DEV)
    H.hdet_quantise_rows(rnd(2, d_out, width), w, ws)
    for r in (5, rows):           # few rows, and tiles
        a, b = torch.empty(2, r, d_out, dtype=BF, device=R.DEV), torch.empty(2, r, d_out, dtype=BF, device=R.DEV)
        s = scale[:, :r].contiguous()
        H.hdet_quantised_linear(codes[:, :r], s, w, ws, a)
        H.hdet_quantised_linear(cf[:, :r], s, w, ws, b)
        assert torch.equal(a, b)
    del cf


def test_loss_with_far_operands():
    g = torch.Generator(device=R.DEV).manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g, device=R.DEV)  # noqa: E731
    for rows, width, classes in ((40, 72, 300), (600, 256, 9000)):
        h, w = rnd(2, rows, width).to(BF), (rnd(2, classes, width) * width ** -0.5).to(BF)
        labels = torch.randint(0, classes, (2, rows), generator=g, device=R.DEV, dtype=torch.int32)

        def call(h, w, dh, dw):
            loss, mean = torch.empty(2, rows, device=R.DEV), torch.empty(2, device=R.DEV)
            work = torch.empty(H.hdet_vocab_loss_workspace(2, rows, width, classes, dw=BF), dtype=torch.uint8, device=R.DEV)
            H.hdet_vocab_loss(h, w, labels, loss, mean, dh=dh, dw=dw, workspace=work)
            return loss, mean, dh, dw
        want = call(h, w, torch.empty_like(h), torch.empty_like(w))
        hf, wf = far(h, True), far(w, True)
        got = call(hf, wf, far(torch.empty_like(h), False), far(torch.empty_like(w), False))
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        del hf, wf, got
        torch.cuda.empty_cache()


def _step(x, r, gain, w, ws, bias, hw, labels, out, work, stream):
    """Norm, 8-bit layer, loss, and back."""
    H.hdet_rmsnorm(x, gain, resid=r, total=out["total"], codes=out["codes"], scale=out["scale"], rstd=out["rstd"], stream=stream)
    H.hdet_quantised_linear(out["codes"], out["scale"], w, ws, out["y"], bias=bias, stream=stream)
    H.hdet_vocab_loss(out["y"], hw, labels, out["loss"], out["mean"], dh=out["dy"], dw=out["dhead"], db=out["dhead_b"], workspace=work, stream=stream)
    H.hdet_quantised_linear_backward(out["dy"], out["codes"], out["scale"], w, ws, dx=out["dn"], dw=out["dw"], db=out["db"], workspace=work, stream=stream)
    H.hdet_rmsnorm_backward(out["total"], gain, out["rstd"], out["dn"], out["dx"], dgain=out["dgain"], workspace=work, stream=stream)


def _problem(n, rows, d, classes, seed):
    g = torch.Generator(device=R.DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=R.DEV)  # noqa: E731
    e = lambda *s, dt=F32: torch.empty(*s, dtype=dt, device=R.DEV)  # noqa: E731
    w, ws = H.hdet_codes_empty(n, d, d), e(n, d)
    H.hdet_quantise_rows(rnd(n, d, d) * d ** -0.5, w, ws)
    args = [rnd(n, rows, d).to(BF), rnd(n, rows, d).to(BF), 1 + 0.1 * rnd(n, d), w, ws, 0.1 * rnd(n, d), (rnd(n, classes, d) * d ** -0.5).to(BF),
            torch.randint(-1, classes, (n, rows), generator=g, device=R.DEV, dtype=torch.int32)]
    out = dict(total=e(n, rows, d, dt=BF), codes=H.hdet_codes_empty(n, rows, d), scale=e(n, rows), rstd=e(n, rows), y=e(n, rows, d, dt=BF), loss=e(n, rows), mean=e(n),
               dy=e(n, rows, d, dt=BF), dhead=e(n, classes, d), dhead_b=e(n, classes), dn=e(n, rows, d, dt=BF), dw=e(n, d, d), db=e(n, d), dx=e(n, rows, d, dt=BF),
               dgain=e(n, d))
    work = torch.empty(max(H.hdet_vocab_loss_workspace(n, rows, d, classes), H.hdet_quantised_linear_backward_workspace(n, rows, d, d),
                           H.hdet_rmsnorm_backward_workspace(n, rows, d)), dtype=torch.uint8, device=R.DEV)
    return args, out, work


@pytest.mark.parametrize("n,rows,d,classes", [(2, 40, 72, 300), (3, 515, 264, 2003), (1, 1100, 512, 20000)])
def test_captured_graph(n, rows, d, classes):
    args, out, work = _problem(n, rows, d, classes, 4)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(*args, out, work, side.cuda_stream)          # (once before, as any program does)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            _step(*args, out, work, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for turn in range(4):
        new = _problem(n, rows, d, classes, 10 + turn)[0]
        for a, b in zip(args, new):
            a.copy_(b)
        for t in out.values():
            t.fill_(7)
        work.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        _step(*args, out, work, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for k in got:
            assert torch.equal(got[k], out[k]), (turn, k)


def test_two_streams_at_once():
    """Calls that share nothing may overlap: two chains on streams of their own against the same chains one after the other."""
    problems = [_problem(2, 300, 136, 1500, s) for s in (1, 2)]
    want = []
    for args, out, work in problems:
        _step(*args, out, work, torch.cuda.current_stream().cuda_stream)
        want.append({k: v.clone() for k, v in out.items()})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    for _ in range(3):
        for (args, out, work), s in zip(problems, streams):
            with torch.cuda.stream(s):
                _step(*args, out, work, s.cuda_stream)
    torch.cuda.synchronize()
    for (_, out, _), w in zip(problems, want):
        assert all(torch.equal(out[k], w[k]) for k in w)
