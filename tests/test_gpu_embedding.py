"""The embedding and the gradient of its table against the formulas in 64 bits.

Tolerances.  U = 2^-24 and B = 2^-8 are the unit roundoffs of fp32 and bf16.  A row of the lookup is rounded once in fp32 and once in its type.  A
sum of n rows in any order of additions is off by n U of the sum of the terms' sizes at most; scaling and adding to what was there are
a rounding each; the type's on top."""
import math

import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _half(dt):
    return 0.0 if dt == torch.float32 else B


def _tokens(kind, K, N, V, g):
    if kind == "one":               # all the same
        tok = torch.full((K, N), V - 1)
    elif kind == "none":
        tok = torch.full((K, N), -1)
    elif kind == "own":             # each its own row, as far as there are enough
        tok = torch.stack([torch.randperm(max(N, V), generator=g)[:N] % V for _ in range(K)])
    elif kind == "zipf":
        tok = (torch.exp(torch.rand(K, N, generator=g, dtype=torch.float64) * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    else:                           # all kinds, outside of the table too
        tok = torch.randint(-2, V + 2, (K, N), generator=g)
        tok.view(-1)[::7] = 2 ** 40
        tok.view(-1)[::11] = -2 ** 62
    return tok.cuda()


def _want(dy, tok, V, scale, old=None):
    """The gradient in 64 bits, and how far it may be off."""
    K, d = tok.shape[0], dy.shape[-1]
    has = (tok >= 0) & (tok < V)
    at = torch.where(has, tok, torch.zeros_like(tok))
    x = torch.where(has[..., None], dy.double(), torch.zeros_like(dy, dtype=torch.float64))
    grad, size, count = (torch.zeros(K, V, n, dtype=torch.float64, device="cuda") for n in (d, d, 1))
    for k in range(K):
        rows = torch.unique(at[k])
        for out, add in ((grad, x[k]), (size, x[k].abs()), (count, has[k].double()[:, None])):
            if len(rows) == 1:          # (index_add_ would wait for itself)
                out[k, rows[0]] = add.sum(0)
            else:
                out[k].index_add_(0, at[k], add)
    want, room = scale * grad, abs(scale) * U * (count + 2) * size
    if old is not None:
        want = want + old.double()
        room = room + torch.where(count > 0, U * (want.abs() + room), torch.zeros_like(room))
    return want, room, count


SIZES = [(1, 1, 1, 1), (1, 4, 9, 7), (2, 5, 3, 8), (1, 100, 40, 9), (3, 65, 513, 64), (1, 1000, 512, 130), (2, 1025, 17, 300), (1, 4096, 700, 24),
         (1, 4097, 700, 24), (2, 9000, 3000, 36), (1, 300, 70000, 12), (1, 5000, 300000, 5), (1, 600, 20, 2100), (1, 40, 11, 9001),
         (2, 2048, 130, 40), (1, 2049, 1000, 16), (1, 1500, 65, 1100), (1, 16384, 40, 9), (2, 17000, 500, 12), (8, 2000, 60000, 4)]


@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("K,N,V,d", SIZES)
def test_lookup(K, N, V, d, table):
    g = torch.Generator().manual_seed(1)
    E = torch.randn(K, V, d, generator=g).to(DT[table]).cuda()
    tok = _tokens("any", K, N, V, g)
    has = ((tok >= 0) & (tok < V))[..., None]
    at = tok.clamp(0, V - 1)
    for out, dt in (("same", DT[table]), ("f32", torch.float32), ("bf16", torch.bfloat16)):
        for scale in (1.0, 11.3):
            y = qsr.embedding(tok, E, scale=scale, out=out)
            s = float(torch.tensor(scale))
            want = torch.where(has, s * torch.stack([E[k][at[k]] for k in range(K)]).double(), torch.zeros((), dtype=torch.float64, device="cuda"))
            assert y.dtype == dt and y.shape == (K, N, d)
            assert (y.double() - want).abs().le((U + _half(dt) * (1 + U)) * want.abs()).all()
    if K == 1:
        assert torch.equal(qsr.embedding(tok.view(-1), E[0], scale=2.0), qsr.embedding(tok, E, scale=2.0)[0])


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("rows", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["any", "one", "own", "zipf", "none"])
@pytest.mark.parametrize("K,N,V,d", SIZES)
def test_gradient(K, N, V, d, kind, rows, grad):
    g = torch.Generator().manual_seed(2)
    tok = _tokens(kind, K, N, V, g)
    dy = torch.randn(K, N, d, generator=g).to(DT[rows]).cuda()
    like = torch.empty(K, V, d, dtype=DT[grad], device="cuda")
    got = qsr.embedding_backward(dy, tok, like, scale=0.7)
    want, room, count = _want(dy, tok, V, float(torch.tensor(0.7)))
    assert got.dtype == DT[grad] and (got.double() - want).abs().le(room + _half(DT[grad]) * (want.abs() + room)).all()
    assert got[(count == 0).expand_as(got)].eq(0).all()
    assert torch.equal(got, qsr.embedding_backward(dy, tok, like, scale=0.7))
    old = torch.randn(K, V, d, generator=g).to(DT[grad]).cuda()
    out = old.clone()
    assert qsr.embedding_backward(dy, tok, like, scale=0.7, out=out, accumulate=True) is out
    want, room, count = _want(dy, tok, V, float(torch.tensor(0.7)), old)
    assert (out.double() - want).abs().le(room + torch.where(count > 0, _half(DT[grad]) * (want.abs() + room), torch.zeros_like(room))).all()
    assert torch.equal(out[(count == 0).expand_as(out)], old[(count == 0).expand_as(old)])


@pytest.mark.parametrize("N,V,d", [(33, 5, 8), (4096, 3, 16), (5000, 2, 8), (20000, 100, 72), (140000, 7, 4)])
def test_whole_numbers_are_summed_exactly(N, V, d):
    """Sums below 2^24 of whole numbers: every term once, wherever chunks and parts of the sort end."""
    g = torch.Generator().manual_seed(3)
    dy = torch.randint(-50, 51, (N, d), generator=g).float().cuda()
    tok = torch.randint(-1, V, (N,), generator=g).cuda()
    got = qsr.embedding_backward(dy, tok, torch.empty(V, d, device="cuda"))
    want = torch.zeros(V + 1, d, dtype=torch.float64, device="cuda").index_add_(0, torch.where(tok < 0, V, tok), dy.double())[:V]
    assert torch.equal(got.double(), want)


def test_gradient_against_differences():
    """The value is linear in the table: a difference of two values is the gradient up to roundings in 64 bits."""
    g = torch.Generator().manual_seed(4)
    V, N, d = 6, 9, 5
    E, dy = torch.randn(V, d, generator=g).cuda(), torch.randn(N, d, generator=g).cuda()
    tok = torch.tensor([0, 5, 5, 2, -1, 6, 5, 0, 3]).cuda()
    got = qsr.embedding_backward(dy, tok, E, scale=1.5)

    def value(E64):
        y = torch.stack([1.5 * E64[t] if 0 <= t < V else torch.zeros_like(E64[0]) for t in tok.tolist()])
        return float((y * dy.double()).sum())
    for j in range(V * d):
        two = []
        for sign in (0.5, -0.5):
            e = E.double().clone()
            e.view(-1)[j] += sign
            two.append(value(e))
        assert abs(two[0] - two[1] - float(got.view(-1)[j])) <= 8 * U * 1.5 * float(dy.abs().sum()) + 1e-12


def test_values_that_are_not_finite_stay_in_their_rows():
    dy = torch.ones(70, 12, device="cuda")
    tok = (torch.arange(70) % 4).cuda()
    dy[5, 3] = float("nan")
    dy[6, 4] = float("inf")
    dy[9] = float("nan")
    tok[9] = -1                     # no token: nothing of its row is taken
    got = qsr.embedding_backward(dy, tok, torch.empty(9, 12, device="cuda"))
    bad = torch.zeros(9, 12, dtype=torch.bool)
    bad[1, 3] = bad[2, 4] = True
    assert torch.equal(~got.isfinite().cpu(), bad) and got[1, 3].isnan() and got[2, 4] == float("inf") and got[4:].eq(0).all()
    table = torch.ones(9, 12, device="cuda")
    table[0] = float("nan")         # what stands in the place of no row is not this one
    y = qsr.embedding(tok, table)
    assert y[9].eq(0).all() and y[0].isnan().all() and y[1].eq(1).all()


def test_strides_and_places():
    """Tables and gradients as parts of wider rows and of workers' flat buffers, rows of y's gradient apart, and another stream."""
    K, N, V, d = 3, 200, 50, 37
    for dt in DT.values():
        g = torch.Generator().manual_seed(5)
        tok = _tokens("any", K, N, V, g)
        E, dy = torch.randn(K, V, d, generator=g).to(dt).cuda(), torch.randn(K, N, d, generator=g).to(dt).cuda()
        y, grad = qsr.embedding(tok, E, scale=3.0), qsr.embedding_backward(dy, tok, E, scale=3.0)
        wide = torch.full((K, V, d + 6), 7.0, dtype=dt, device="cuda")
        flat = torch.full((K, V * d + 11), 7.0, dtype=dt, device="cuda")
        apart = torch.full((K, N, d + 3), float("nan"), dtype=dt, device="cuda")[..., 1:1 + d]
        apart.copy_(dy)
        for view in (wide[..., 1:1 + d], flat[:, 3:3 + V * d].view(K, V, d)):
            view.copy_(E)
            assert torch.equal(qsr.embedding(tok, view, scale=3.0), y)
            assert qsr.embedding_backward(apart, tok, E, scale=3.0, out=view) is view and torch.equal(view, grad)
        assert wide[..., 0].eq(7).all() and wide[..., 1 + d:].eq(7).all() and flat[:, :3].eq(7).all() and flat[:, 3 + V * d:].eq(7).all()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        a, b = qsr.embedding(tok, E, scale=3.0, stream=side.cuda_stream), qsr.embedding_backward(dy, tok, E, scale=3.0, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(a, y) and torch.equal(b, grad)


def test_nothing():
    E = torch.ones(5, 8, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert qsr.embedding(none, E).shape == (0, 8)
    assert qsr.embedding_backward(torch.empty(0, 8, device="cuda"), none, E).eq(0).all()
    out = E.clone()
    assert qsr.embedding_backward(torch.empty(0, 8, device="cuda"), none, E, out=out, accumulate=True).eq(1).all()
    one = torch.tensor(3, device="cuda")
    assert qsr.embedding(one, E, scale=2.0).eq(2).all() and qsr.embedding(one, E).shape == (8,)


def test_recorded_and_replayed():
    """Small and large sorts; tokens change between the replays."""
    g = torch.Generator().manual_seed(6)
    for N, V in ((500, 90), (6000, 9000)):
        E, dy = torch.randn(2, V, 24, generator=g).cuda(), torch.randn(2, N, 24, generator=g).cuda()
        tok = _tokens("zipf", 2, N, V, g)
        qsr.embedding_backward(dy, tok, E)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, grad = qsr.embedding(tok, E), qsr.embedding_backward(dy, tok, E)
        for kind in ("zipf", "any", "one"):
            tok.copy_(_tokens(kind, 2, N, V, g))
            want = qsr.embedding(tok, E), qsr.embedding_backward(dy, tok, E)
            y.zero_(), grad.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want[0]) and torch.equal(grad, want[1])


def test_refusals():
    E, tok = torch.ones(2, 5, 8, device="cuda"), torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    dy = torch.ones(2, 3, 8, device="cuda")
    for call in (lambda: qsr.embedding(tok.int(), E), lambda: qsr.embedding(tok.cpu(), E), lambda: qsr.embedding(tok, E.half()),
                 lambda: qsr.embedding(tok[:1], E), lambda: qsr.embedding(tok[:, ::2], E), lambda: qsr.embedding(tok, E[0, 0]),
                 lambda: qsr.embedding(tok, E.transpose(1, 2)), lambda: qsr.embedding_backward(dy[..., :7], tok, E),
                 lambda: qsr.embedding_backward(dy[:1], tok, E), lambda: qsr.embedding_backward(dy.double(), tok, E),
                 lambda: qsr.embedding_backward(dy, tok, E, accumulate=True), lambda: qsr.embedding_backward(dy, tok, E, out=E[:, :4]),
                 lambda: qsr.embedding_backward(dy, tok, E, out=E.half()), lambda: qsr.embedding_backward(dy, tok, E, out=E.cpu())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(qsr.QSRError):       # workers' gradients on top of each other
        qsr.embedding_backward(dy, tok, E, out=torch.ones(1, 5, 8, device="cuda").expand(2, 5, 8))
    with pytest.raises(qsr.QSRError):
        qsr.embedding(tok, E, scale=float("nan"))
