"""The operators over more rows than they have workgroups: the norm's backward pass with several trips to every workgroup, and log
probabilities of more rows than a grid's second dimension holds."""
import pytest
import torch

import paper_2310_14423_amd as qsr
from test_gpu_rmsnorm import DT, U, _data, _half
from test_gpu_token_logprobs import _logits

pytestmark = pytest.mark.gpu

# (rows, d): two to four trips to each of the workgroups that a worker's rows get, and not the same number to all.  One size for
# every way in which a row is shared out among lanes (fp32 and bf16 part from 512 on).
TRIPS = [(40965, 2), (45001, 7), (41003, 96), (61447, 128), (20489, 200), (5003, 500), (6143, 768), (2501, 1003), (1301, 2048), (1537, 4096),
         (601, 8192), (771, 16383)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 3])
@pytest.mark.parametrize("rows,d", TRIPS)
def test_norm_backward_with_several_trips(rows, d, K, dt):
    """Tolerances as for few rows: the row's sum is off by 32 U of its terms' sizes, the weight's gradient by (rows + 4) U."""
    dt = DT[dt]
    x, res, w, dy, dres = _data(K, rows, d, dt, 11)
    f = qsr.rmsnorm(x, w, residual=res, eps=1e-6)
    dx, dw = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, residual_grad=dres)
    for k in range(K):
        r = f.rstd[k].double()[:, None]
        n, y = f.sum[k].double() * r, dy[k].double()
        u = y * w[k].double()
        mean, size = (u * n).mean(-1, keepdim=True), (u * n).abs().mean(-1, keepdim=True)
        want, down = r * (u - n * mean) + dres[k].double(), dres[k].double()
        room = r * (6 * U * u.abs() + n.abs() * (40 * U * size + 6 * U * mean.abs())) + 2 * U * (want.abs() + down.abs())
        assert (dx[k].double() - want).abs().le(room + _half(dt) * (want.abs() + room)).all()
        terms = y * n
        assert (dw[k].double() - terms.sum(0)).abs().le((rows + 4) * U * terms.abs().sum(0)).all()
    again = qsr.rmsnorm_backward(dy, f.sum, w, f.rstd, residual_grad=dres)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V,top", [(70, 3), (70, 0), (300, 20), (2500, 2), (2500, 64)])
def test_more_rows_than_a_grid_has(V, top, dt):
    """Rows in one call, and the same in two that a grid can hold, each long enough to be shared out alike: the same bits."""
    n = 70001
    x, tok = _logits(n, V, DT[dt], V + top)
    x[::7, ::3] = -torch.inf
    x[5::11, 1::2] = torch.finfo(DT[dt]).min
    x[65537], tok[65539] = -torch.inf, -1
    a, b = torch.linspace(-1, 1, n, device="cuda"), torch.linspace(2, -1, n, device="cuda")
    f = qsr.token_logprobs(x, tok, top=top)
    d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, a, b)
    for part in (slice(0, 33000), slice(33000, n)):
        y, t = x[part], tok[part]
        g = qsr.token_logprobs(y, t, top=top)
        for s, u in zip(f, g):
            assert s is None if u is None else torch.equal(s[part], u)
        assert torch.equal(d[part], qsr.token_logprobs_backward(y, t, g.stats, g.entropy, a[part], b[part]))
