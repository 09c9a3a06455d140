"""Log probabilities of given tokens, entropy, alternatives and their gradient against the formulas in 64 bits.

Tolerances.  U = 2^-24.  A lane adds at most c = V / 64 + 8 terms one after the other and the lanes are joined in a tree (12 more);
a term's exponent is off by a rounding of its size, which the term's own weight e^-t keeps below one unit, and the exponential by
two: the sum s is off by D = (c + 20) U relative at most, hence log s by D.  lse has a rounding of its own size more, log
probabilities those of x - m and of the result.  The entropy is log s - w / s with |w| / s <= log s + (the entropy): D (2 + 2 (H + log s)).
A gradient entry is p times a sum whose terms' sizes are |a| and |b| (|log p| + H): p is off by D + 4 U (1 + |log p|) relative; the
entropy's own error enters through H.  bf16 results (eight significant bits) have a rounding of 2^-8 more."""
import numpy as np
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _logits(rows, V, dt, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, V, generator=g) * spread).to(dt)
    return x.cuda(), torch.randint(0, V, (rows,), generator=g).cuda()


def _exact(x, tok, T):
    z = x.double().cpu() / T
    top = z.amax(-1)
    rel = z - top.clamp_min(-1e300)[:, None]        # (taken from the maximum: 64 bits too lose log s beside the lowest float)
    ls = rel.exp().sum(-1).log()
    lse, lp = top + ls, rel - ls[:, None]
    lp[lse == -np.inf] = -np.inf
    p = lp.exp()
    H = -torch.where(p > 0, p * lp, 0 * p).sum(-1)
    tok = tok.cpu()
    has = (tok >= 0) & (tok < x.shape[1])
    logp = torch.where(has, lp.gather(1, torch.where(has, tok, 0 * tok)[:, None])[:, 0], 0 * lse)
    ls[lse == -np.inf] = 0
    return z, lp, p, H, logp, lse, has, ls


def _order(x, k):
    v = torch.where(x.isnan(), torch.full_like(x, -np.inf), x).float().cpu().numpy()
    return np.argsort(-v, axis=-1, kind="stable")[:, :k]


def _close(got, want, room):
    got, want = got.double().cpu(), want.double()
    same = got == want          # infinities
    assert (same | ((got - want).abs() <= room)).all(), float((got - want).abs().nan_to_num(0, 0, 0).max())


def _check(x, tok, k, T):
    f = qsr.token_logprobs(x, tok, top=k, temperature=T)
    z, lp, p, H, logp, lse, has, ls = _exact(x, tok, T)
    V = x.shape[1]
    D = (V / 64 + 28) * U
    fin = lambda t: t.nan_to_num(0, 0, 0).abs()  # noqa: E731
    _close(f.lse, lse, D + 2 * U * fin(lse) + 2 * U * fin(z.amax(-1)))
    _close(f.entropy, H, D * (2 + 2 * (H + ls)))
    _close(f.logp, logp, D + 4 * U * fin(logp))
    if k:
        at = _order(x, k)
        assert np.array_equal(f.top_id.cpu().numpy(), at)
        want = lp.gather(1, torch.from_numpy(at))
        _close(f.top_logp, want, (D + 4 * U * fin(want)))
    else:
        assert f.top_logp is None and f.top_id is None
    return f


SIZES = [(1, 1), (1, 2), (3, 5), (2, 63), (2, 65), (5, 255), (4, 1000), (2, 1023), (3, 2048), (2, 4100), (1, 8193), (2, 16383), (3, 33001),
         (1, 131072), (1, 200003), (600, 3001), (520, 9000), (1030, 300)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", SIZES)
def test_forward(rows, V, dt):
    x, tok = _logits(rows, V, DT[dt], rows + V)
    for k in {0, 1, min(V, 7), min(V, 64)}:
        _check(x, tok, k, 1.0)
    _check(x, tok, min(V, 3), 0.7)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 3000, 50000])
def test_masks(V, dt):
    """-inf and the type's lowest value as masks: some, all but one, all; tokens that are masked or none."""
    dt = DT[dt]
    x, tok = _logits(9, V, dt, V)
    low = torch.finfo(dt).min
    x[0, ::2] = -np.inf
    x[1, 1::3] = low
    x[2] = -np.inf
    x[3] = low
    x[4] = -np.inf
    x[4, V - 2] = -5.0
    x[5, :V - 1] = low
    x[6, tok[6]] = -np.inf
    x[7] = low
    x[7, 3:9] = -np.inf
    tok[8] = -1
    tok[1] = V
    for k in (0, 5, 20):
        f = _check(x, tok, k, 1.0)
    assert f.lse[2] == -np.inf and f.logp[2] == -np.inf and f.entropy[2] == 0
    assert f.top_id[2].tolist() == list(range(20)) and f.top_logp[2].eq(-np.inf).all()
    assert abs(f.logp[3].item() + np.log(V)) < 1e-4 and abs(f.entropy[3].item() - np.log(V)) < 1e-4
    assert f.logp[8] == 0 and f.logp[1] == 0 and f.entropy[4] == 0
    g = torch.full((9,), 2.0, device="cuda")
    d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, g, g).float()
    assert d.isfinite().all() and d[2].eq(0).all() and d[4].eq(torch.where(torch.arange(V, device="cuda") == tok[4], 2.0, 0.0) -
                                                              torch.where(torch.arange(V, device="cuda") == V - 2, 2.0, 0.0)).all()


@pytest.mark.parametrize("V", [64, 5000, 40000])
def test_ties_and_orders(V):
    """Equal logits, ascending and descending rows, both zeros: the alternatives are the first ones."""
    x = torch.zeros(6, V)
    x[0] = 1.5
    x[1] = torch.arange(V) / 7
    x[2] = -torch.arange(V) / 7
    x[3] = torch.arange(V) % 3
    x[4, 1::2] = -0.0
    x[5] = (torch.arange(V) // 8 % 2).float()
    tok = torch.arange(6).cuda()
    for dt in DT.values():
        for k in (1, 8, 33, 64):
            _check(x.to(dt).cuda(), tok, k, 1.0)


def test_alternatives_in_few_places():
    """More logits above the bound than the kernel's list holds: the largest ones all lie in the lanes that own the bound."""
    V = 400000
    x = torch.full((600, V), -3.0)          # rows enough for a workgroup of 512 lanes each; a lane takes four logits at a time
    x[:2] = torch.randn(2, V, generator=torch.Generator().manual_seed(1))
    lane = torch.arange(V) // 4 % 512
    x[:2, lane < 63] += 50.0
    x[:2, lane == 63] = 40.0
    x = x.cuda()
    tok = torch.zeros(600, dtype=torch.int64, device="cuda")
    f = qsr.token_logprobs(x, tok, top=64)
    assert np.array_equal(f.top_id[:2].cpu().numpy(), _order(x[:2], 64))
    assert np.array_equal(f.top_id[2:].cpu().numpy(), np.tile(np.arange(64), (598, 1)))


def test_rows_that_are_not_finite():
    x, tok = _logits(4, 3000, torch.float32, 3)
    x[0, 17] = np.nan
    x[1, 5] = np.inf
    x[2, :4] = np.nan
    f = qsr.token_logprobs(x, tok, top=6)
    for t in (f.logp, f.entropy, f.lse):
        assert t[:3].isnan().all() and t[3].isfinite()
    assert np.array_equal(f.top_id.cpu().numpy(), _order(x, 6))
    assert f.top_logp[:3].isnan().all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", SIZES)
def test_backward(rows, V, dt):
    dt = DT[dt]
    x, tok = _logits(rows, V, dt, rows * V)
    if rows > 2:
        tok[1] = -1
        x[2, ::2] = -np.inf
    gen = torch.Generator().manual_seed(5)
    a, b = torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()
    for T in (1.0, 1.7):
        f = qsr.token_logprobs(x, tok, temperature=T)
        z, lp, p, H, logp, lse, has, ls = _exact(x, tok, T)
        for ga, gb in ((a, b), (a, None), (None, b)):
            d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, ga, gb, temperature=T)
            A = ga.double().cpu()[:, None] if ga is not None else torch.zeros(rows, 1, dtype=torch.float64)
            Bt = gb.double().cpu()[:, None] if gb is not None else 0 * A
            A = A * has[:, None]
            lpz = torch.where(p > 0, lp, torch.zeros_like(lp))
            want = -p * (A + Bt * (lpz + H[:, None]))
            want.scatter_add_(1, torch.where(has, tok.cpu(), 0 * tok.cpu())[:, None], A)
            D = (V / 64 + 28) * U
            size = A.abs() + Bt.abs() * (lpz.abs() + H[:, None])
            room = p * size * (D + 8 * U * (1 + lpz.abs())) + p * Bt.abs() * D * (2 + 2 * (H + ls)[:, None]) + 2 * U * want.abs()
            want, room = want / T, room / T
            assert d.dtype == dt
            _close(d, want, room * 1.01 + 1e-37 + (B * want.abs() if dt == torch.bfloat16 else 0))


def test_gradient_against_differences():
    """Central differences, in 64 bits, of sum(a logp + b H): truncation and cancellation are below 1e-9, the gradient is fp32."""
    x, tok = _logits(3, 11, torch.float32, 8, 1.0)
    tok[2] = -1
    a, b, T, h = torch.tensor([0.7, -1.3, 2.0]), torch.tensor([0.4, 1.1, -0.6]), 1.3, 1e-5
    f = qsr.token_logprobs(x, tok, temperature=T)
    d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, a.cuda(), b.cuda(), temperature=T)

    def value(y):
        _, _, _, H, logp, _, _, _ = _exact(y, tok, T)
        return float((a.double() * logp + b.double() * H).sum())
    for i in range(x.numel()):
        two = []
        for s in (h, -h):
            y = x.double().cpu()
            y.view(-1)[i] += s
            two.append(value(y))
        assert abs((two[0] - two[1]) / (2 * h) - float(d.view(-1)[i])) <= 2e-6


def test_strides_and_places():
    """Rows out of a wider buffer at any element, the gradient in the logits' place, leading dimensions, another stream."""
    for dt in DT.values():
        for V in (77, 5001):
            x, tok = _logits(6, V, dt, V)
            g = torch.linspace(-1, 1, 6, device="cuda")
            wide = torch.zeros(6, V + 33, dtype=dt, device="cuda")[:, 3:3 + V]
            wide.copy_(x)
            f, h = qsr.token_logprobs(x, tok, top=5), qsr.token_logprobs(wide, tok, top=5)
            assert torch.equal(f.top_id, h.top_id)
            for s, t in zip(f[:4], h[:4]):      # another alignment: other lanes add the terms
                assert (s - t).abs().le((V / 64 + 28) * 40 * U).all()
            d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, g, g)
            out = torch.zeros(6, V + 7, dtype=dt, device="cuda")[:, 2:2 + V]
            e = qsr.token_logprobs_backward(wide, tok, f.stats, f.entropy, g, g, out=out)
            assert e is out and torch.equal(d, e)
            y = x.clone()
            qsr.token_logprobs_backward(y, tok, f.stats, f.entropy, g, g, out=y)
            assert torch.equal(y, d)
            h = qsr.token_logprobs(x.view(2, 3, V), tok.view(2, 3), top=5)
            assert h.logp.shape == (2, 3) and h.top_id.shape == (2, 3, 5) and torch.equal(h.logp.view(6), f.logp)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            h = qsr.token_logprobs(x, tok, top=5, stream=side.cuda_stream)
            e = qsr.token_logprobs_backward(x, tok, h.stats, h.entropy, g, g, stream=side.cuda_stream)
            side.synchronize()
            assert torch.equal(h.logp, f.logp) and torch.equal(h.top_id, f.top_id) and torch.equal(e, d)


def test_recorded_and_replayed():
    x, tok = _logits(3, 70000, torch.bfloat16, 9)
    want = qsr.token_logprobs(x, tok, top=4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = qsr.token_logprobs(x, tok, top=4)
    for _ in range(3):
        for t in f:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(f, want))
        torch.randn(1000, device="cuda").sum().item()


def test_offsets_beyond_32_bits():
    """Rows whose elements lie beyond 2^32 bytes and 2^31 elements from the first."""
    V = 1 << 20
    buf = torch.zeros(2100 * V, dtype=torch.bfloat16, device="cuda")
    x = buf.view(2100, V)
    x[-1] = torch.randn(V, device="cuda").to(torch.bfloat16)
    tok = torch.full((2100,), 5, dtype=torch.int64, device="cuda")
    f = qsr.token_logprobs(x, tok, top=2)
    z, lp, p, H, logp, lse, has, ls = _exact(x[-1:], tok[-1:], 1.0)
    assert abs(float(f.logp[-1]) - float(logp)) < 1e-3 and f.top_id[-1].tolist() == _order(x[-1:], 2)[0].tolist()
    assert abs(float(f.logp[-2]) + np.log(V)) < 1e-3
    d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, torch.ones(2100, device="cuda"), out=x)
    assert abs(float(d[-1, 5]) - (1 - float(p[0, 5]))) < 5e-3 and abs(float(d[0, 7]) * V + 1) < 5e-3


def test_no_rows_and_limits():
    x, tok = torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    f = qsr.token_logprobs(x, tok, top=3)
    assert f.logp.shape == (0,) and f.top_id.shape == (0, 3)
    assert qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, f.logp).shape == (0, 50)
    x, tok = _logits(2, 100, torch.float32, 1)
    for top, code in ((65, -7), (-1, -1), (101, -1)):
        with pytest.raises(qsr.QSRError) as e:
            qsr.token_logprobs(x, tok, top=top)
        assert e.value.code == code
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(qsr.QSRError):
            qsr.token_logprobs(x, tok, temperature=bad)
    with pytest.raises(ValueError):
        qsr.token_logprobs(x, tok.int())
    with pytest.raises(ValueError):
        qsr.token_logprobs(x.half(), tok)
