"""Rows of zeros, and rows whose squares vanish in fp32, where eps does not keep the root away from zero (0, or nothing as a float): they
have rstd 0, are zeros like a row of zeros with any eps, and leave the weight's gradient to the other rows."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [5, 100, 700, 3001, 9000])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-60, 1.5e-45, 1e-30])
def test_rows_of_zeros(eps, dt, d):
    g = torch.Generator().manual_seed(d)
    x = torch.randn(2, 6, d, generator=g).to(dt).cuda()
    w, dy = (1 + 0.1 * torch.randn(2, d, generator=g)).cuda(), torch.randn(2, 6, d, generator=g).to(dt).cuda()
    x[0, 2], x[1, 5], x[1, 0] = 0, 0, 1e-30
    zero = torch.zeros(2, 6, dtype=torch.bool, device="cuda")
    zero[0, 2] = zero[1, 5] = True
    if eps < 1e-50:
        zero[1, 0] = True
    f = qsr.rmsnorm(x, w, eps=eps)
    q = qsr.rmsnorm(x, w, eps=eps, out="fp8")
    assert f.y.isfinite().all() and f.rstd.isfinite().all() and f.y[zero].eq(0).all()
    if eps < 1e-50:
        assert f.rstd[zero].eq(0).all()
    assert q.y.float().isfinite().all() and q.y[zero].float().eq(0).all() and q.scale[zero].eq(0).all() and torch.equal(q.rstd, f.rstd)
    dx, dw = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, residual_grad=dy)
    assert dx.isfinite().all() and dw.isfinite().all()
    if eps < 1e-50:
        assert torch.equal(dx[zero], dy[zero])
    # the other rows and the weight's gradient are those of the rows without these
    for k in range(2):
        keep = ~zero[k]
        alone = qsr.rmsnorm(x[k][keep], w[k], eps=eps)
        assert torch.equal(alone.y, f.y[k][keep]) and torch.equal(alone.rstd, f.rstd[k][keep])
        n = f.sum[k][keep].double() * f.rstd[k][keep].double()[:, None]
        terms = dy[k][keep].double() * n
        assert (dw[k].double() - terms.sum(0)).abs().le(10 * 2.0 ** -24 * terms.abs().sum(0)).all()      # six rows: (rows + 4) U
