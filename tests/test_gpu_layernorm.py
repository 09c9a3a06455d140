"""Layer norm with the residual's addition against the formulas in 64 bits.

Tolerances.  U = 2^-24 is the unit roundoff of fp32, B = 2^-8 that of bf16 (eight significant bits).  A mean over d terms, each lane adding at most
sixteen of them and the lanes in a tree, is off by 30 U of the mean of the terms' sizes at most, its quotient included.  So s - mean is off by
delta = U |s| + 30 U mean|s| + U |s - mean|, the mean of its square by 2 mean(|s - mean| delta) + mean(delta^2) and 30 U of itself, rstd relatively by
half of that and 4 U; y has delta, rstd's error, and four roundings of its own.  In the backward pass the two sums of a row are off by (30 + 4) U of the
mean of their terms' sizes, and the sums over rows by (rows + 4) U of the sum of theirs.  What is stored in bf16 has its rounding on top."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _half(dt):
    return 0.0 if dt == torch.float32 else B


def _data(K, rows, d, dt, seed):
    """Rows whose means are some tenths of their deviation, of sizes that differ."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x, res = r(K, rows, d).to(dt).cuda(), ((r(K, rows, d) + 0.3 * r(K, rows, 1)) * torch.exp(r(K, rows, 1))).to(dt).cuda()
    return x, res, (1 + 0.2 * r(K, d)).cuda(), (0.3 * r(K, d)).cuda(), r(K, rows, d).to(dt).cuda(), r(K, rows, d).to(dt).cuda()


def _forward64(x, res, w, b, eps=EPS):
    """The sum, mean, rstd and y, and how far mean, rstd (relatively) and y may be off."""
    s = x.double() + (res.double() if res is not None else 0)
    size = s.abs().mean(-1, keepdim=True)
    mean = s.mean(-1, keepdim=True)
    v = s - mean
    var = v.pow(2).mean(-1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    delta = U * s.abs() + 30 * U * size + U * v.abs()
    off = (2 * (v.abs() * delta).mean(-1, keepdim=True) + delta.pow(2).mean(-1, keepdim=True) + 30 * U * var) / (2 * (var + eps)) + 4 * U
    n = v * rstd * w.double()[:, None]
    y = n + (b.double()[:, None] if b is not None else 0)
    room = (n.abs() * (off + 4 * U) + delta * rstd * w.double()[:, None].abs()) * (1 + 64 * U) + U * y.abs()
    return s, mean[..., 0], rstd[..., 0], y, 31 * U * size[..., 0], off[..., 0], room


SIZES = [(1, 1, 1), (1, 1, 7), (2, 3, 64), (1, 5, 511), (3, 4, 512), (2, 2, 513), (1, 9, 768), (2, 3, 1003), (1, 2, 1024), (1, 3, 1025),
         (1, 2, 2049), (2, 2, 4096), (1, 2, 4097), (1, 1, 8192), (1, 2, 8195), (1, 1, 16384), (2, 700, 96), (1, 1300, 130)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", SIZES)
def test_forward(K, rows, d, dt):
    dt = DT[dt]
    x, res, w, b, _, _ = _data(K, rows, d, dt, 1)
    for r, bias in ((res, b), (res, None), (None, b), (None, None)):
        f = qsr.layernorm(x, w, bias, residual=r, eps=EPS)
        s, mean, rstd, y, d_mean, d_rstd, room = _forward64(x, r, w, bias)
        assert f.scale is None and f.y.dtype == dt and f.rstd.shape == f.mean.shape == (K, rows)
        if r is None:
            assert f.sum is x
        else:
            assert f.sum.dtype == dt and (f.sum.double() - s).abs().le((U + _half(dt)) * s.abs()).all()
        assert (f.mean.double() - mean).abs().le(d_mean).all()
        assert (f.rstd.double() - rstd).abs().le(d_rstd * rstd).all()
        assert (f.y.double() - y).abs().le(room + _half(dt) * (y.abs() + room)).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", SIZES)
def test_codes(K, rows, d, dt):
    """Codes are the e4m3 values nearest to y / scale, up to y's error, with scale = max|y| / 448."""
    x, res, w, b, _, _ = _data(K, rows, d, DT[dt], 2)
    f = qsr.layernorm(x, w, b, residual=res, eps=EPS, out="fp8")
    _, mean, rstd, y, d_mean, d_rstd, room = _forward64(x, res, w, b)
    assert f.y.dtype == torch.float8_e4m3fn and f.scale.shape == (K, rows)
    assert (f.mean.double() - mean).abs().le(d_mean).all() and (f.rstd.double() - rstd).abs().le(d_rstd * rstd).all()
    top, off = y.abs().amax(-1), room.amax(-1)
    assert (f.scale.double() - top / 448).abs().le((off + 4 * U * top) / 448).all()
    v = y / (top / 448)[..., None]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    slack = (room + v.abs() / 448 * off[..., None]) / (top / 448)[..., None] + 8 * U * v.abs()
    # (an error that carries v over a border of two steps may meet the wider one)
    assert (f.y.double() - v).abs().le(0.5 * step + slack * (1 + 2.0 ** -3)).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", SIZES)
def test_backward(K, rows, d, dt):
    dt = DT[dt]
    x, res, w, b, dy, dres = _data(K, rows, d, dt, 3)
    f = qsr.layernorm(x, w, b, residual=res, eps=EPS)
    rs, mu = f.rstd.double()[..., None], f.mean.double()[..., None]
    n, u = (f.sum.double() - mu) * rs, dy.double() * w.double()[:, None]
    p, q, sp, sq = (t.mean(-1, keepdim=True) for t in (u, u * n, u.abs(), (u * n).abs()))
    for down, bias in ((dres, True), (None, False)):
        dx, dw, db = qsr.layernorm_backward(dy, f.sum, w, f.mean, f.rstd, residual_grad=down, bias=bias)
        want = rs * (u - p - n * q)
        room = rs * (8 * U * (u.abs() + p.abs() + (n * q).abs()) + 34 * U * (sp + n.abs() * sq))
        if down is not None:
            want = want + down.double()
            room = room + 2 * U * (want.abs() + down.double().abs())
        assert dx.dtype == dt and (dx.double() - want).abs().le(room + _half(dt) * (want.abs() + room)).all()
        terms = dy.double() * n
        assert dw.dtype == torch.float32 and (dw.double() - terms.sum(1)).abs().le((rows + 4) * U * terms.abs().sum(1)).all()
        if bias:
            assert db.dtype == torch.float32 and (db.double() - dy.double().sum(1)).abs().le((rows + 4) * U * dy.double().abs().sum(1)).all()
        else:
            assert db is None


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,d", [(6, 90, 1100), (1, 3, 1536), (2, 2, 1537), (1, 40, 2048), (1, 3, 2560), (1, 2, 2561), (5, 90, 4204), (1, 3, 5120), (1, 2, 5121),
                                      (2, 3, 9001), (6, 50, 12288), (1, 2, 12289), (3, 701, 1003), (7, 1000, 64), (3, 500, 700)])
def test_more_widths(K, rows, d, dt):
    """Widths between the powers of two; rows enough for several to a workgroup, and workers that do not divide the chip."""
    test_forward(K, rows, d, dt)
    test_codes(K, rows, d, dt)
    test_backward(K, rows, d, dt)


@pytest.mark.parametrize("K,rows,d", [(1, 1, 5), (2, 3, 17)])
def test_gradient_against_differences(K, rows, d):
    """Central differences, in 64 bits, of sum(y * dy) + sum(s * dres): truncation h^2 = 1e-10, cancellation 1e-16 / h = 1e-11,
    both times sums of some tens of terms of size one and rstd's third power, below a hundred here; the gradient itself is fp32."""
    x, res, w, b, dy, dres = _data(K, rows, d, torch.float32, 4)
    f = qsr.layernorm(x, w, b, residual=res, eps=EPS)
    grads = qsr.layernorm_backward(dy, f.sum, w, f.mean, f.rstd, residual_grad=dres)

    def value(x64, w64, b64):
        s = x64 + res.double()
        v = s - s.mean(-1, keepdim=True)
        y = v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w64[:, None] + b64[:, None]
        return float((y * dy.double()).sum() + (s * dres.double()).sum())
    h = 1e-5
    for i, got in enumerate(grads):
        at = [x.double(), w.double(), b.double()]
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
        x, res, w, b, dy, dres = _data(K, rows, d, dt, 5)
        wide = [torch.zeros(K, rows, d + 40, dtype=dt, device="cuda")[..., o:o + d] for o in (1, 3, 5, 7)]
        for v, t in zip(wide, (x, res, dy, dres)):
            v.copy_(t)
        apart = [torch.full((K, d + 9), float("nan"), device="cuda")[:, o:o + d] for o in (2, 3)]
        apart[0].copy_(w)
        apart[1].copy_(b)
        f = qsr.layernorm(x, w, b, residual=res)
        for args in ((wide[0], w, b, wide[1]), (x, apart[0], apart[1], res)):
            g = qsr.layernorm(*args[:3], residual=args[3])
            assert all(torch.equal(p, q) for p, q in zip(f[:4], g[:4]))
        back = qsr.layernorm_backward(dy, f.sum, w, f.mean, f.rstd, dres)
        again = qsr.layernorm_backward(wide[2], f.sum, apart[0], f.mean, f.rstd, wide[3])
        assert all(torch.equal(p, q) for p, q in zip(back, again))
        for out, other in ((res.clone(), x), (x.clone(), res)):
            h = qsr.layernorm(out, w, b, residual=other, sum_out=out)
            assert h.sum is out and torch.equal(out, f.sum) and torch.equal(h.y, f.y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        h = qsr.layernorm(x, w, b, residual=res, stream=side.cuda_stream)
        again = qsr.layernorm_backward(dy, h.sum, w, h.mean, h.rstd, dres, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(h.y, f.y) and all(torch.equal(p, q) for p, q in zip(back, again))


@pytest.mark.parametrize("d", [70, 3000])
def test_rows_out_of_the_ordinary(d):
    """Equal numbers, a mean far above the deviation, numbers whose squares leave fp32 at either end, and rows that are not finite, beside
    an ordinary row."""
    g = torch.Generator().manual_seed(6)
    w, b = torch.ones(d, device="cuda"), torch.full((d,), 0.25, device="cuda")
    x = torch.randn(7, d, generator=g).cuda()
    x[1] = 3.0
    x[2] = 4096.0 + torch.randint(-2, 3, (d,), generator=g).cuda()             # sums below 2^24: the mean is off by its rounding alone
    x[3] *= 1e-30
    x[4, 7] = float("nan")
    x[5, 9] = float("inf")
    x[6] *= 1e30
    f, q = qsr.layernorm(x, w, b, eps=EPS), qsr.layernorm(x, w, b, eps=EPS, out="fp8")
    assert f.mean[1] == 3 and f.y[1].eq(0.25).all() and f.rstd[1].sub(EPS ** -0.5).abs() < 1e-3
    _, mean, rstd, y, d_mean, d_rstd, room = _forward64(x[None, :4], None, w[None], b[None])
    assert (f.y[:4].double() - y[0]).abs().le(room[0]).all() and (f.rstd[:4].double() - rstd[0]).abs().le(d_rstd[0] * rstd[0]).all()
    # 4096 + small: 2^-12 of the mean's rounding against a deviation of 1.4
    assert (f.y[2].double() - y[0, 2]).abs().max() < 1e-3
    for t in (f.y[4], f.y[5], q.y[4].float(), q.y[5].float()):
        assert t.isnan().all()
    assert f.rstd[4].isnan() and f.rstd[5].isnan() and f.rstd[6] == 0 and f.y[6].eq(0.25).all()
    none = qsr.layernorm(x[1:2], w, b, eps=0.0)
    assert none.rstd[0] == 0 and none.y.eq(0.25).all()
    dx, _, _ = qsr.layernorm_backward(torch.ones_like(x[1:2]), x[1:2], w, none.mean, none.rstd)
    assert dx.eq(0).all()


def test_no_rows_and_single_rows():
    w, b = torch.ones(40, device="cuda"), torch.zeros(40, device="cuda")
    nothing = torch.empty(0, 40, device="cuda")
    f = qsr.layernorm(nothing, w, b, out="fp8")
    assert f.y.shape == (0, 40) and f.scale.shape == f.mean.shape == (0,)
    dx, dw, db = qsr.layernorm_backward(nothing, nothing, w, f.mean, f.rstd)
    assert dx.shape == (0, 40) and dw.eq(0).all() and db.eq(0).all()
    x = torch.arange(40.0, device="cuda")
    f = qsr.layernorm(x, w, eps=0.0)
    assert f.y.shape == (40,) and f.rstd.shape == () and f.mean == 19.5


def test_recorded_and_replayed():
    x, res, w, b, dy, dres = _data(2, 60, 200, torch.bfloat16, 7)
    want = qsr.layernorm(x, w, b, residual=res)
    back = qsr.layernorm_backward(dy, want.sum, w, want.mean, want.rstd, dres)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = qsr.layernorm(x, w, b, residual=res)
        g = qsr.layernorm_backward(dy, f.sum, w, f.mean, f.rstd, dres)
    for _ in range(3):
        for t in (*f[:4], *g):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((*f[:4], *g), (*want[:4], *back)))
        torch.randn(1000, device="cuda").sum().item()


def test_many_rows():
    """More rows than there are workgroups, in the widest and the narrowest layout: each as if it were alone."""
    for rows, d in ((70000, 24), (1500, 9000)):
        g = torch.Generator().manual_seed(8)
        x = torch.randn(rows, d, generator=g).cuda()
        w, b = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
        f = qsr.layernorm(x, w, b, out="fp8")
        for i in (0, rows // 2, rows - 1):
            one = qsr.layernorm(x[i:i + 1], w, b, out="fp8")
            assert torch.equal(one.y.view(torch.uint8), f.y[i:i + 1].view(torch.uint8)) and torch.equal(one.scale, f.scale[i:i + 1])


def test_limits():
    x, w = torch.zeros(1, 16385, device="cuda"), torch.ones(16385, device="cuda")
    with pytest.raises(qsr.QSRError) as e:
        qsr.layernorm(x, w)
    assert e.value.code == -7
    ok = torch.zeros(4, 8, device="cuda")
    v = torch.ones(8, device="cuda")
    n = torch.zeros(4, device="cuda")
    for call in (lambda: qsr.layernorm(ok.half(), v), lambda: qsr.layernorm(ok, v[:3]), lambda: qsr.layernorm(ok, v, v[:3]),
                 lambda: qsr.layernorm(ok, v, v.bfloat16()), lambda: qsr.layernorm(ok, v, v.cpu()), lambda: qsr.layernorm(torch.zeros(8, 8, device="cuda").t(), v),
                 lambda: qsr.layernorm(ok, v.expand(4, 8), v), lambda: qsr.layernorm(ok, v, residual=ok.bfloat16()),
                 lambda: qsr.layernorm_backward(ok, ok, v, n, n[:3]), lambda: qsr.layernorm_backward(ok, ok, v, n.double(), n),
                 lambda: qsr.layernorm_backward(ok[:3], ok, v, n, n)):
        with pytest.raises(ValueError):
            call()
