"""Layer norm, the embedding and the gated recurrence where offsets pass 31 and 32 bits: the same as side by side, and nothing else is
written.  (Buffers of some GB, of which little is used.)"""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
FAR = (1 << 31) + 4096          # elements


def _apart(t, stride, first=8):
    """t's rows along its first dimension, `stride` elements apart."""
    flat = torch.empty(stride * (t.shape[0] - 1) + t[0].numel() + 2 * first, dtype=t.dtype, device="cuda")
    view = torch.as_strided(flat, t.shape, (stride,) + t.stride()[1:], first)
    view.copy_(t)
    return view


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_layernorm(dt):
    g = torch.Generator().manual_seed(1)
    x, dy = torch.randn(3, 100, generator=g).to(dt).cuda(), torch.randn(3, 100, generator=g).to(dt).cuda()
    w, b = torch.ones(100, device="cuda"), torch.zeros(100, device="cuda")
    f = qsr.layernorm(x, w, b)
    far = _apart(x, FAR)
    n = qsr.layernorm(far, w, b)
    assert all(torch.equal(p, q) for p, q in zip((f.y, f.mean, f.rstd), (n.y, n.mean, n.rstd)))
    want = qsr.layernorm_backward(dy, x, w, f.mean, f.rstd, residual_grad=dy)
    got = qsr.layernorm_backward(dy, far, w, f.mean, f.rstd, residual_grad=dy)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [40, 3000, 20000])
def test_embedding(dt, N):
    """A table of more than 2^32 bytes, and one whose rows are as far apart; workers too."""
    g = torch.Generator().manual_seed(2)
    V, d = (FAR // 1024) + 3, 1024
    table = torch.empty(V, d, dtype=dt, device="cuda")
    tok = torch.randint(V - 50, V + 1, (N,), generator=g).cuda()
    rows = torch.randn(50, d, generator=g).to(dt).cuda()
    table[-50:] = rows
    dy = torch.randn(N, d, generator=g).to(dt).cuda()
    y = qsr.embedding(tok, table)
    near = torch.where(tok < V, tok - (V - 50), -1)
    assert torch.equal(y, qsr.embedding(near, rows))
    # sums of whole numbers are the same in any order, whatever way is taken
    dy = (dy * 4).round()
    want = qsr.embedding_backward(dy, near, rows, out=torch.empty(50, d, device="cuda"))
    if dt == torch.float32:
        grad = qsr.embedding_backward(dy, tok, table, out=table)
        assert torch.equal(grad[-50:], want) and grad[0].eq(0).all() and grad[V // 2].eq(0).all() and grad[-51].eq(0).all()
        grad[:4] = 7
    else:
        grad = table
        grad[:4] = 7
        grad[-50:] = 0
    qsr.embedding_backward(dy, tok, table, out=grad, accumulate=True)
    twice = 2 * want if dt == torch.float32 else want.to(dt)
    assert torch.equal(grad[-50:], twice) and grad[:4].eq(7).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 9, 40])
def test_sequences_far_apart(dt, T):
    g = torch.Generator().manual_seed(3)
    x, f, dh = (torch.randn(3, T, 33, generator=g).to(dt).cuda() for _ in range(3))
    s = qsr.gated_scan(x, f, keep=True)
    far = _apart(x, FAR)
    n = qsr.gated_scan(far, f, keep=True)
    assert all(torch.equal(p, q) for p, q in zip(s, n))
    want, got = qsr.gated_scan_backward(dh, x, f, s.states), qsr.gated_scan_backward(dh, far, f, s.states)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_steps_far_apart(dt):
    """As far as they may be; further is refused."""
    g = torch.Generator().manual_seed(4)
    x, f, dh = (torch.randn(1, 150, 40, generator=g).to(dt).cuda() for _ in range(3))
    s = qsr.gated_scan(x, f, keep=True)
    far = _apart(x[0], 1 << 24)[None]
    n = qsr.gated_scan(far, f, keep=True)
    assert all(torch.equal(p, q) for p, q in zip(s, n))
    want, got = qsr.gated_scan_backward(dh, x, f, s.states), qsr.gated_scan_backward(dh, far, f, s.states)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    del far, n, got
    with pytest.raises(qsr.QSRError) as e:
        qsr.gated_scan(_apart(x[0, :3], (1 << 24) + 1)[None], f[:, :3])
    assert e.value.code == -7


def test_long_and_many():
    """More than 2^31 elements in all: the last sequence is as it is alone."""
    B, T, d = 9, 4096, 65536
    x = torch.empty(B, T, d, dtype=torch.bfloat16, device="cuda")
    for b in (0, B - 1):
        x[b].normal_(generator=torch.Generator(device="cuda").manual_seed(b))
    x[1:-1] = 0
    f = qsr.gated_scan(x, x)
    for b in (0, B - 1):
        one = qsr.gated_scan(x[b:b + 1], x[b:b + 1])
        # (alone it is shared out in other ways)
        assert (f.last[b] - one.last[0]).abs().max() <= 2.0 ** -14 and (f.h[b, -1].float() - one.h[0, -1].float()).abs().max() <= 2.0 ** -5
    assert f.h[3, -1].eq(0).all()
