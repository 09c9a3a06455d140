"""The root-mean-square norm with the residual's addition against the formulas in 64 bits.

Tolerances.  U = 2^-24 is the unit roundoff of fp32, B = 2^-8 that of bf16 (eight significant bits).  A mean over d squares, each lane adding at most
sixteen of them and the lanes in a tree, is off by (16 + 12) U relative at most, its root by half of that plus two roundings; y has
two more.  24 U covers rstd and y.  In the backward pass the row's sum is off by (16 + 12 + 4) U of the sum of its terms' sizes, and
the weight's gradient by (rows + 4) U of the sum of its terms' sizes.  What is stored in bf16 has its rounding on top."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _half(dt):
    return 0.0 if dt == torch.float32 else B


def _data(K, rows, d, dt, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x, res = (r(K, rows, d) * spread).to(dt).cuda(), (r(K, rows, d) * torch.exp(r(K, rows, 1))).to(dt).cuda()
    return x, res, (1 + 0.2 * r(K, d)).cuda(), r(K, rows, d).to(dt).cuda(), r(K, rows, d).to(dt).cuda()


def _forward64(x, res, w, eps):
    s = x.double() + (res.double() if res is not None else 0)
    rstd = 1 / (s.pow(2).mean(-1) + eps).sqrt()
    return s, rstd, s * rstd[..., None] * w.double()[:, None]


SIZES = [(1, 1, 1), (1, 1, 7), (2, 3, 64), (1, 5, 511), (3, 4, 512), (2, 2, 513), (1, 9, 768), (2, 3, 1003), (1, 2, 1024), (1, 3, 1025),
         (1, 2, 2049), (2, 2, 4096), (1, 2, 4097), (1, 1, 8192), (1, 2, 8195), (1, 1, 16384), (2, 700, 96), (1, 1300, 130)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", SIZES)
def test_forward(K, rows, d, dt):
    dt = DT[dt]
    x, res, w, _, _ = _data(K, rows, d, dt, 1)
    f = qsr.rmsnorm(x, w, residual=res, eps=1e-6)
    s, rstd, y = _forward64(x, res, w, 1e-6)
    assert f.scale is None and f.y.dtype == dt and f.sum.dtype == dt and f.rstd.shape == (K, rows)
    assert (f.sum.double() - s).abs().le((U + _half(dt)) * s.abs()).all()
    assert (f.rstd.double() - rstd).abs().le(24 * U * rstd).all()
    assert (f.y.double() - y).abs().le((24 * U + _half(dt) * (1 + 24 * U)) * y.abs()).all()
    # without a residual the sum is x itself, and nothing is written for it
    f = qsr.rmsnorm(x, w, eps=1e-6)
    s, rstd, y = _forward64(x, None, w, 1e-6)
    assert f.sum is x and (f.y.double() - y).abs().le((24 * U + _half(dt) * (1 + 24 * U)) * y.abs()).all()


def _assert_nearest(codes, scale, y):
    """Codes are the e4m3 values nearest to y / scale, up to 2^-18 of a step, with scale = max|y| / 448."""
    top = y.abs().amax(-1)
    assert (scale.double() - top / 448).abs().le(32 * U * top / 448 + 1e-45).all()
    v = y / (top / 448).clamp_min(1e-300)[..., None]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    assert (codes.double() - v).abs().le(step * (0.5 + 2.0 ** -18) + 40 * U * v.abs()).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", SIZES)
def test_codes(K, rows, d, dt):
    x, res, w, _, _ = _data(K, rows, d, DT[dt], 2)
    f = qsr.rmsnorm(x, w, residual=res, out="fp8")
    _, rstd, y = _forward64(x, res, w, 1e-6)
    assert f.y.dtype == torch.float8_e4m3fn and f.scale.shape == (K, rows)
    assert (f.rstd.double() - rstd).abs().le(24 * U * rstd).all()
    _assert_nearest(f.y, f.scale, y)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", SIZES)
def test_backward(K, rows, d, dt):
    dt = DT[dt]
    x, res, w, dy, dres = _data(K, rows, d, dt, 3)
    f = qsr.rmsnorm(x, w, residual=res, eps=1e-6)
    for down in (dres, None):
        dx, dw = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, residual_grad=down)
        n, u = f.sum.double() * f.rstd.double()[..., None], dy.double() * w.double()[:, None]
        mean, size = (u * n).mean(-1, keepdim=True), (u * n).abs().mean(-1, keepdim=True)
        want = f.rstd.double()[..., None] * (u - n * mean)
        room = f.rstd.double()[..., None] * (6 * U * u.abs() + n.abs() * (40 * U * size + 6 * U * mean.abs()))
        if down is not None:
            want = want + down.double()
            room = room + 2 * U * (want.abs() + down.double().abs())
        assert dx.dtype == dt and (dx.double() - want).abs().le(room + _half(dt) * (want.abs() + room)).all()
        terms = dy.double() * n
        assert dw.dtype == torch.float32 and (dw.double() - terms.sum(1)).abs().le((rows + 4) * U * terms.abs().sum(1)).all()


@pytest.mark.parametrize("K,rows,d", [(1, 1, 5), (2, 3, 17)])
def test_gradient_against_differences(K, rows, d):
    """Central differences, in 64 bits, of sum(y * dy) + sum(s * dres): truncation h^2 = 1e-10, cancellation 1e-16 / h = 1e-11,
    both times sums of some tens of terms of size one; the gradient itself is fp32."""
    x, res, w, dy, dres = _data(K, rows, d, torch.float32, 4)
    f = qsr.rmsnorm(x, w, residual=res, eps=1e-6)
    dx, dw = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, residual_grad=dres)

    def value(x64, w64):
        s = x64 + res.double()
        y = s / (s.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w64[:, None]
        return float((y * dy.double()).sum() + (s * dres.double()).sum())
    h = 1e-5
    for got, i in ((dx, 0), (dw, 1)):
        at = [x.double(), w.double()]
        scale = float(got.abs().max())
        for j in range(got.numel()):
            two = []
            for sign in (1, -1):
                arg = [t.clone() for t in at]
                arg[i].view(-1)[j] += sign * h
                two.append(value(*arg))
            assert abs((two[0] - two[1]) / (2 * h) - float(got.view(-1)[j])) <= 1e-5 * (1 + scale)


def test_strides_and_places():
    """Rows out of a wider buffer that start at any element, inputs and outputs in the same memory, and another stream."""
    K, rows, d = 2, 5, 333
    for dt in DT.values():
        x, res, w, dy, dres = _data(K, rows, d, dt, 5)
        wide = [torch.zeros(K, rows, d + 40, dtype=dt, device="cuda")[..., o:o + d] for o in (1, 3, 5, 7)]
        for v, t in zip(wide, (x, res, dy, dres)):
            v.copy_(t)
        f, g = qsr.rmsnorm(x, w, residual=res), qsr.rmsnorm(wide[0], w, residual=wide[1])
        assert torch.equal(f.y, g.y) and torch.equal(f.sum, g.sum) and torch.equal(f.rstd, g.rstd)
        apart = torch.full((K, d + 9), float('nan'), device='cuda')[:, 2:2 + d]
        apart.copy_(w)
        g = qsr.rmsnorm(x, apart, residual=res)
        assert torch.equal(f.y, g.y)
        a, b = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, dres), qsr.rmsnorm_backward(wide[2], f.sum, apart, f.rstd, wide[3])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        for out in (res.clone(), x.clone()):
            other = res if torch.equal(out, x) else x
            h = qsr.rmsnorm(out, w, residual=other, sum_out=out)
            assert h.sum is out and torch.equal(out, f.sum) and torch.equal(h.y, f.y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        h = qsr.rmsnorm(x, w, residual=res, stream=side.cuda_stream)
        b = qsr.rmsnorm_backward(dy, h.sum, w, h.rstd, dres, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(h.y, f.y) and torch.equal(b[0], a[0]) and torch.equal(b[1], a[1])


def test_rows_out_of_the_ordinary():
    """Rows of zeros, of numbers whose squares leave the small end of fp32, and rows that are not finite, beside an ordinary one."""
    d = 70
    w = torch.ones(d, device="cuda")
    x = torch.randn(5, d, generator=torch.Generator().manual_seed(6)).cuda()
    x[1] = 0
    x[2] *= 1e-30
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    f, q = qsr.rmsnorm(x, w, eps=1e-6), qsr.rmsnorm(x, w, eps=1e-6, out="fp8")
    assert f.y[1].eq(0).all() and f.rstd[1].sub(1e3).abs() < 1e-3
    assert torch.allclose(f.y[2], x[2] * 1e3, rtol=1e-6, atol=0)
    assert f.y[3].isnan().all() and f.rstd[3].isnan()
    assert f.y[4, 9].isnan() and f.y[4, :9].eq(0).all() and f.rstd[4] == 0
    assert q.y[1].float().eq(0).all() and q.scale[1] == 0
    assert q.y[3].float().isnan().all() and q.y[4, 9].float().isnan() and q.y[4, 10:].float().eq(0).all()
    s, _, y = _forward64(x[None, :1], None, w[None], 1e-6)
    _assert_nearest(q.y[:1], q.scale[:1], y[0])
    assert f.y[0].sub(y[0, 0]).abs().le(24 * U * y[0, 0].abs()).all()


def test_no_rows_and_single_rows():
    w = torch.ones(40, device="cuda")
    f = qsr.rmsnorm(torch.empty(0, 40, device="cuda"), w, out="fp8")
    assert f.y.shape == (0, 40) and f.scale.shape == (0,)
    dx, dw = qsr.rmsnorm_backward(torch.empty(0, 40, device="cuda"), torch.empty(0, 40, device="cuda"), w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 40) and dw.eq(0).all()
    f = qsr.rmsnorm(torch.ones(40, device="cuda"), w, eps=0.0)
    assert f.y.shape == (40,) and f.rstd.shape == () and f.y.eq(1).all()


def test_recorded_and_replayed():
    x, res, w, dy, dres = _data(2, 60, 200, torch.bfloat16, 7)
    want = qsr.rmsnorm(x, w, residual=res)
    back = qsr.rmsnorm_backward(dy, want.sum, w, want.rstd, dres)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = qsr.rmsnorm(x, w, residual=res)
        b = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, dres)
    for _ in range(3):
        for t in (*f[:3], *b):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(f.y, want.y) and torch.equal(b[0], back[0]) and torch.equal(b[1], back[1])
        torch.randn(1000, device="cuda").sum().item()


def test_limits():
    x = torch.zeros(1, 16385, device="cuda")
    with pytest.raises(qsr.QSRError) as e:
        qsr.rmsnorm(x, torch.ones(16385, device="cuda"))
    assert e.value.code == -7
    with pytest.raises(ValueError):
        qsr.rmsnorm(x.half(), torch.ones(16385, device="cuda"))
    with pytest.raises(ValueError):
        qsr.rmsnorm(x, torch.ones(3, device="cuda"))
    with pytest.raises(ValueError):
        qsr.rmsnorm(torch.zeros(8, 8, device="cuda").t(), torch.ones(8, device="cuda"))
