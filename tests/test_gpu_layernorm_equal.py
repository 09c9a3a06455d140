"""Layer norm of rows whose numbers are all the same: no deviation, whatever the sum of the row was rounded to.  The mean is the number, y is
the bias, rstd is 1 / sqrt(eps), or 0 without eps, and then the row has no gradient.  All of that is exact: the tolerances are zero, but for
rstd's, 4 roundings."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
NUMBERS = [0.1, 1 / 3, -0.7, 1.0000001, 1234.567, -7.7e5, 3.3e-7, 1.7e12, 0.0]


@pytest.mark.parametrize("d", [3, 7, 100, 257, 511, 768, 1003, 1537, 2200, 4204, 5120, 8191, 9001, 12000, 16384])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_fp32(d, eps):
    x = torch.tensor(NUMBERS, device="cuda")[:, None].expand(-1, d).contiguous()
    g = torch.Generator().manual_seed(d)
    w, b = torch.randn(d, generator=g).cuda(), torch.randn(d, generator=g).cuda()
    f = qsr.layernorm(x, w, b, eps=eps)
    assert torch.equal(f.mean, x[:, 0])
    assert torch.equal(f.y, b.expand_as(x))
    if eps == 0.0:
        assert f.rstd.eq(0).all()
        down = torch.randn(len(NUMBERS), d, generator=g).cuda()
        dx, dw, _ = qsr.layernorm_backward(down, x, w, f.mean, f.rstd, residual_grad=down)
        assert torch.equal(dx, down) and dw.eq(0).all()
    else:
        assert f.rstd.sub(eps ** -0.5).abs().le(4 * 2.0 ** -24 * eps ** -0.5).all()


@pytest.mark.parametrize("d", [7, 768, 1003, 4204, 16384])
def test_sums_of_bf16(d):
    """x + residual has more digits than either: its row is equal numbers all the same."""
    x = torch.tensor(NUMBERS, device="cuda").bfloat16()[:, None].expand(-1, d).contiguous()
    res = torch.tensor([1.1, -300.0, 0.003, 5.0, 0.07, 12.0, 9.0, 3.0, 0.0], device="cuda").bfloat16()[:, None].expand(-1, d).contiguous()
    w, b = torch.ones(d, device="cuda"), torch.linspace(-2, 2, d, device="cuda")
    f = qsr.layernorm(x, w, b, residual=res, eps=0.0)
    assert torch.equal(f.mean, (x.float() + res.float())[:, 0]) and f.rstd.eq(0).all()
    assert torch.equal(f.y, b.bfloat16().expand_as(x))


@pytest.mark.parametrize("d", [64, 1003, 4204])
def test_means_far_above_the_deviation(d):
    """One step of the floats around a large number: the deviation is half a step, and is found to 2^-10 of itself.  (The numbers less
    the sum's quotient are whole steps, a few tens at most, as exact as their squares; so y keeps what mean, rounded, cannot.)"""
    n = 2 * (d // 2)
    x = torch.full((4, n), 3.0e6, device="cuda")
    x[:, ::2] += 0.25
    w = torch.ones(n, device="cuda")
    f = qsr.layernorm(x, w, eps=0.0)
    assert f.rstd.sub(8.0).abs().le(8.0 * 2.0 ** -10).all()
    assert f.y[:, ::2].sub(1.0).abs().le(2.0 ** -10).all() and f.y[:, 1::2].add(1.0).abs().le(2.0 ** -10).all()
