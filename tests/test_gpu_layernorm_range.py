"""Layer norm of finite rows whose sums leave the range of fp32, while no number is further than the largest float from the mean: the square of the
deviation is infinite, so rstd is 0, y is the bias, and the row has no gradient; all of that is exact.  The mean is off by 31 roundings of the
mean of the sizes."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _check(x, res=None):
    d = x.shape[-1]
    g = torch.Generator().manual_seed(d)
    w, b, down = torch.randn(d, generator=g).cuda(), torch.randn(d, generator=g).cuda(), torch.randn(len(x), d, generator=g).to(x.dtype).cuda()
    s = x.double() if res is None else x.double() + res.double()
    f = qsr.layernorm(x, w, b, residual=res, eps=1e-5)
    assert (f.mean.double() - s.mean(-1)).abs().le(31 * U * s.abs().mean(-1)).all()
    assert f.rstd.eq(0).all() and torch.equal(f.y, b.to(x.dtype).expand_as(x))
    dx, dw, db = qsr.layernorm_backward(down, f.sum, w, f.mean, f.rstd, residual_grad=down)
    assert torch.equal(dx, down) and dw.eq(0).all() and (db.double() - down.double().sum(0)).abs().le(len(x) * U * down.double().abs().sum(0)).all()
    q = qsr.layernorm(x, w, b, residual=res, eps=1e-5, out="fp8")
    assert torch.equal(q.scale, (b.abs().amax() * torch.tensor(1 / 448.0)).expand(len(x))) and q.y.float().isfinite().all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [2, 100, 250, 768, 1003, 1600, 4204, 12000, 16384])
def test_large_numbers(d, dt):
    """Around a mean, spread about zero, and of two sizes."""
    g = torch.Generator().manual_seed(d + 1)
    r = torch.rand(4, d, generator=g) - 0.5
    r[:, 0], r[:, 1] = -0.5, 0.5            # (rows that are not equal numbers)
    x = torch.stack([3e34 + 2e34 * r[0], 1e38 + 1e38 * r[1], 3.3e38 * r[2], 1.6e38 * torch.sign(r[3])]).to(dt).cuda()
    _check(x)
    _check((0.25 * x.float()).to(dt), (0.5 * x.float()).to(dt).flip(-1))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [768, 1024])
def test_lowest_numbers_beside_ordinary_ones(d, dt):
    x = torch.randn(2, d, generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    x[0, d // 2:] = torch.finfo(dt).min
    x[1, 5] = torch.finfo(dt).min
    _check(x)
