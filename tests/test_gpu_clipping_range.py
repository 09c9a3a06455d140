"""Clipping by global norm where it can go wrong: gradients whose squares leave the range of fp32, gradients that are not finite, and
lists on either side of the number of partial sums that the update adds up itself (64).

Tolerances.  U = 2^-24.  The norm of a list is exact to its own rounding, U: squares and sums are double.  The factor is rounded once;
its 1e-6 is exact.  m after one step from zero is (1 - beta1) coef g: four roundings (the factor's, the product's, that of 1 - beta1 and
the result's), 6 U allowed; v is (1 - beta2)(coef g)^2: those of coef g count twice, and three more, 10 U allowed."""
import ctypes as C

import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8


def _factors(opt):
    """The K factors and norms of the last step, copied from the library's arrays."""
    coef, norm = C.c_void_p(), C.c_void_p()
    assert qsr.lib().qsr_adamw_clip(opt._handle, C.byref(coef), C.byref(norm)) == 0

    class Floats:
        def __init__(self, address, n):
            self.__cuda_array_interface__ = dict(shape=(n,), typestr="<f4", data=(address, False), version=3)
    torch.cuda.synchronize()
    return tuple(torch.as_tensor(Floats(p.value, opt.K), device="cuda").clone().cpu() for p in (coef, norm))


def _gradients(sizes, K, gtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(K, n, generator=g) * 10.0 ** (-i % 3)).to(gtype).cuda() for i, n in enumerate(sizes)]


def _step(grads, states, clip):
    params = [torch.zeros(g.shape, device="cuda") for g in grads]
    opt = qsr.AdamW(params, grads, states=states, beta1=B1, beta2=B2, eps=EPS, clip_norm=clip)
    opt.step(1e-2, 0)
    return params, opt


def _norm64(grads):
    return torch.stack([sum(g[k].double().pow(2).sum() for g in grads).sqrt() for k in range(len(grads[0]))]).cpu()


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["f32", "fp8"])
@pytest.mark.parametrize("where", [0, 70], ids=["one partial sum", "many"])
@pytest.mark.parametrize("size", [2e19, 1e20, 3e38, 1e-25])
def test_squares_outside_fp32(size, where, states, gtype):
    """A finite gradient whose square is not: the norm and the factor are finite all the same, and what is left of the others is
    scaled by it; a worker of gradients whose squares vanish has a norm too."""
    sizes = [300, 5] + [17] * where
    g = _gradients(sizes, 2, gtype, 1)
    if size < 1:
        for x in g:
            x[1] *= size
    else:
        g[-1][1, 3] = size
    norm = _norm64(g)
    clip = float(norm[0]) * 0.5
    want = (clip / (norm + 1e-6)).clamp(max=1.0)
    _, opt = _step(g, states, clip)
    coef, got = _factors(opt)
    assert (got.double() - norm).abs().le(2 * U * norm).all(), (got, norm)
    assert (coef.double() - want).abs().le(2 * U * want + 1e-45).all(), (coef, want)
    if states == "f32":
        for i, x in enumerate(g):
            m = (1 - B1) * want[:, None].cuda() * x.double()
            assert (opt.m[i].double() - m).abs().le(6 * U * m.abs() + 1e-44).all()


@pytest.mark.parametrize("states", ["f32", "fp8"])
@pytest.mark.parametrize("where", [0, 70], ids=["one partial sum", "many"])
def test_gradients_that_are_not_finite(where, states):
    """An infinite gradient makes the norm infinite and the factor 0: its element is spoilt, the others' gradients count as zero.  One
    that is no number leaves no norm to clip by: factor 1, its element is spoilt, the others are stepped as they are."""
    g = _gradients([300, 9] + [20] * where, 3, torch.float32, 2)
    last = len(g) - 1
    g[last][1, 4], g[last][2, 4] = float("inf"), float("nan")
    clip = float(_norm64(g)[0]) * 0.5
    p, opt = _step(g, states, clip)
    coef, norm = _factors(opt)
    assert coef[1] == 0 and norm[1] == float("inf") and coef[2] == 1 and norm[2].isnan() and abs(float(coef[0]) - 0.5) < 1e-5
    alone, other = _step(g, states, 0.0)
    for i, x in enumerate(p):
        keep = torch.ones(x.shape[1], dtype=torch.bool, device="cuda")
        if i == last:
            keep[4] = False
            assert x[1:, 4].isnan().all() and x[0].isfinite().all()
        assert x[1][keep].eq(0).all() and torch.equal(x[2][keep], alone[i][2][keep])
        m, n = opt.moments(i)[0], other.moments(i)[0]
        assert m[1][keep].eq(0).all() and torch.equal(m[2][keep], n[2][keep])


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[5] * 63, [5] * 64, [5] * 65, [70, 16385] * 40, [3], [64 * 16384], [64 * 16384 + 1], [5000011, 3],
                                   [70000003, 7]], ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_factors_of_any_list(sizes, gtype):
    """Up to 64 partial sums, more, and spans longer than 64 blocks: norms, factors and the moments that come of them."""
    K = 2
    g = _gradients([min(n, 1 << 20) for n in sizes], K, gtype, 3)
    g = [x if x.shape[1] == n else x.repeat(1, n // x.shape[1] + 1)[:, :n].contiguous() for x, n in zip(g, sizes)]
    for x in g:
        x[1] *= 2.0 ** -8
    norm = _norm64(g)
    clip = float(norm[0]) * 0.25
    want = (clip / (norm + 1e-6)).clamp(max=1.0)
    assert want[1] == 1
    _, opt = _step(g, "f32", clip)
    coef, got = _factors(opt)
    assert (got.double() - norm).abs().le(2 * U * norm).all() and (coef.double() - want).abs().le(2 * U * want).all()
    for i, x in enumerate(g):
        m = (1 - B1) * want[:, None].cuda() * x.double()
        v = (1 - B2) * (want[:, None].cuda() * x.double()).pow(2)
        assert (opt.m[i].double() - m).abs().le(6 * U * m.abs()).all() and (opt.v[i].double() - v).abs().le(10 * U * v + 1e-44).all()


def test_codes_of_a_long_clipped_list():
    """More than 64 partial sums with 8-bit moments: the scales are those of the scaled gradients (from zero: m = (1 - beta1) coef g),
    within the roundings of m and four of their own."""
    g = _gradients([300] * 70, 2, torch.bfloat16, 4)
    norm = _norm64(g)
    clip = float(norm.min()) * 0.125
    want = clip / (norm + 1e-6)
    _, opt = _step(g, "fp8", clip)
    for i in (0, 33, 69):
        x = torch.nn.functional.pad(g[i].double(), (0, 212)).view(2, 2, 256).abs().amax(-1) * want[:, None].cuda()
        for scale, top in ((opt.m_scale[i], (1 - B1) * x), (opt.v_scale[i], (1 - B2) ** 0.5 * x)):
            assert (scale.double() * 448 - top).abs().le(12 * U * top).all()


@pytest.mark.parametrize("at", [0, 2, 500, -1])
@pytest.mark.parametrize("K,P", [(3, 5), (2, 1027), (3, 20001), (2, 300003)])
def test_flat_rows_outside_fp32(K, P, at):
    """Flat rows: one element of row 1 whose square is no float, infinite or no number, wherever it lies in the row.  Ordinary rows'
    norms are off by the roundings of the squares, U at most; a factor may be subnormal."""
    at = min(at, P - 1)
    g = torch.randn(K, P, generator=torch.Generator().manual_seed(5)).cuda()
    plain = qsr.clip_factors(g, 1.5)
    for size, infinite in ((2e19, False), (-3e38, False), (float("inf"), True), (float("nan"), None)):
        g[1, at] = size
        norm = g.double().pow(2).sum(1).sqrt().cpu()
        for coef, got in (qsr.clip_factors(g, 1.5), _static_factors(g, 1.5)):
            coef, got = coef.cpu(), got.cpu()
            for k in range(K):
                if k != 1:
                    assert coef[k] == plain[0][k] and got[k] == plain[1][k]
                    assert abs(float(got[k]) - float(norm[k])) <= 4 * U * float(norm[k])
                elif infinite is None:
                    assert coef[1] == 1 and got[1].isnan()
                elif infinite:
                    assert coef[1] == 0 and got[1] == float("inf")
                else:
                    want = 1.5 / (float(norm[1]) + 1e-6)
                    assert abs(float(got[1]) - float(norm[1])) <= 4 * U * float(norm[1]) and abs(float(coef[1]) - want) <= 4 * U * want + 1e-45


def _static_factors(g, clip):
    out = torch.empty(2, g.shape[0], device="cuda")
    qsr.clip_factors_static(g, clip, out[0], out[1])
    return out[0], out[1]
