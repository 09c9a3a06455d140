"""AdamW over many tensors against the formulas in 64 bits, and against the [K][P] update of a context, bit for bit.

Tolerances.  U = 2^-24.  m and v take two roundings of the size of their terms, 4 U (|m| + |g|); the step m / (r + eps) six more;
the parameter one of its own size.  8-bit moments: a block's scale is off by 4 U relative; a code is the value below or above
x / scale and the one that the step's random words choose, except where x / scale plus the word lies within 2^-14 of a step, and the
moment's own error (of the size of its terms, which may cancel) of a border: sixteen steps of x, off by 8 U and 2^-22, are 2^-16."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2310_14423_amd as qsr
import workloads

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8
SETS = [[1], [7], [255, 256, 257], [1024, 1025, 3], [5000, 17, 4096, 1], [100003, 64], [3] * 300, [2, 700001]]


def _tensors(sizes, K, gtype, seed, scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    p = [torch.randn(K, n, generator=g).cuda() for n in sizes]
    grads = [(torch.randn(K, n, generator=g) * scale * 10.0 ** (-i % 3)).to(gtype).cuda() for i, n in enumerate(sizes)]
    return p, grads


def _step64(p, g, m, v, eta, t, lam, coef=1.0):
    g = g.double() * coef
    m = m + (1 - B1) * (g - m)
    v = v + (1 - B2) * (g * g - v)
    upd = eta * (m / (1 - B1 ** (t + 1))) / ((v / (1 - B2 ** (t + 1))).sqrt() + EPS)
    return p.double() - eta * lam * p.double() - upd, m, v, upd


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 3])
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_moments_in_32_bits(sizes, K, gtype):
    p, g = _tensors(sizes, K, gtype, 1)
    lam = [0.05 if i % 2 else 0.0 for i in range(len(sizes))]
    copies = [torch.zeros_like(x, dtype=torch.bfloat16) for x in p]
    opt = qsr.AdamW(p, g, copies=copies, weight_decay=lam, beta1=B1, beta2=B2, eps=EPS)
    want = [[x.clone(), torch.zeros_like(x, dtype=torch.float64), torch.zeros_like(x, dtype=torch.float64)] for x in p]
    for t in range(3):
        before = [x.clone() for x in p]
        opt.step(1e-2, t)
        for i, x in enumerate(p):
            th, m, v, upd = _step64(before[i], g[i], want[i][1], want[i][2], 1e-2, t, lam[i])
            want[i][1:] = [m, v]
            gd = g[i].double().abs()
            assert (opt.m[i].double() - m).abs().le(6 * (t + 1) * U * (m.abs() + gd)).all()
            assert (opt.v[i].double() - v).abs().le(6 * (t + 1) * U * (v.abs() + gd * gd)).all()
            assert (x.double() - th).abs().le(2 * U * th.abs() + 40 * (t + 1) * U * upd.abs() + 1e-12).all()
            assert torch.equal(copies[i], x.to(torch.bfloat16))


def test_the_bits_of_a_context():
    """One tensor [K][P] with fp32 moments: parameters and moments of a context's own update."""
    for P in (20004, 5003, 3001):
        w = workloads.get("flat60m", K=4, P=P, T=20, model="external", power=0, H_base=100)
        th0 = np.random.default_rng(0).standard_normal(P).astype(np.float32)
        ctx = qsr.Context(w, theta0=th0)
        p, g = ctx.params.clone(), torch.zeros_like(ctx.grads)
        opt = qsr.AdamW([p], [g], weight_decay=w["lam"], beta1=w["beta1"], beta2=w["beta2"], eps=w["eps"])
        eta = ctx.eta_table()
        for t in range(5):
            g.copy_(torch.randn(4, P, generator=torch.Generator().manual_seed(t)) * 1e-2)
            ctx.grads.copy_(g)
            ctx.local_step()
            ctx.maybe_sync()
            opt.step(float(eta[t]), t)
        assert torch.equal(ctx.params, p) and torch.equal(ctx.state0, opt.m[0]) and torch.equal(ctx.state1, opt.v[0])
        ctx.close()


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["f32", "fp8"])
@pytest.mark.parametrize("sizes", [[5], [300, 20000, 1], [70001, 3, 16384, 40000]], ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_clipping_over_the_list(sizes, states, gtype):
    """Norms over all tensors of a worker, a worker above the threshold and one below; the step is that of the scaled gradients."""
    K = 3
    p, g = _tensors(sizes, K, gtype, 2)
    for x in g:
        x[1] *= 1e-3
    norm = torch.stack([sum(x[k].double().pow(2).sum() for x in g).sqrt() for k in range(K)])
    c = float(norm[0]) * 0.25
    coef = (c / (norm + 1e-6)).clamp(max=1.0)
    assert coef[1] == 1 and coef[0] < 0.3
    q = [x.clone() for x in p]
    opt = qsr.AdamW(p, g, states=states, beta1=B1, beta2=B2, eps=EPS, clip_norm=c)
    opt.step(1e-2, 0)
    for i in range(len(sizes)):
        th, _, _, upd = _step64(q[i], g[i], 0.0, 0.0, 1e-2, 0, 0.0, coef[:, None])
        assert (p[i].double() - th).abs().le(2 * U * th.abs() + 60 * U * upd.abs() + 1e-7 * upd.abs()).all()
    ptr, ptr2 = C.c_void_p(), C.c_void_p()
    assert qsr.lib().qsr_adamw_clip(opt._handle, C.byref(ptr), C.byref(ptr2)) == 0 and ptr.value and ptr2.value


def _word(seed, t):
    z = (seed + (t + 1) * 0x9E3779B97F4A7C15) & (2 ** 64 - 1)
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & (2 ** 64 - 1)
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & (2 ** 64 - 1)
    return (z ^ (z >> 31)) >> 32


def _fractions(seed, t, k, first, n):
    x = (np.arange(first, first + n, dtype=np.uint64) + np.uint64(k * 0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    x ^= np.uint64(_word(seed, t))
    M = np.uint64(0xFFFFFFFF)
    x ^= x >> np.uint64(16); x = x * np.uint64(0x21F0AAAD) & M
    x ^= x >> np.uint64(15); x = x * np.uint64(0x735A2D97) & M
    x ^= x >> np.uint64(15)
    return (x >> np.uint64(16)).astype(float) / 65536, (x & np.uint64(0xFFFF)).astype(float) / 65536


def _check_codes(code, scale, x, size, u, positive):
    """code, scale of one worker's tensor, padded; x: the exact values, `size` that of their terms; u: the
    fractions that round them."""
    n = len(x)
    nb = -(-n // 256)
    pad = np.zeros(nb * 256)
    pad[:n] = x
    top = np.abs(pad.reshape(nb, 256)).max(1)
    top[top < 1e-35] = 0
    assert np.all(np.abs(scale - top / 448) <= 4 * U * top / 448)
    y = pad / np.repeat(np.where(top > 0, top / 448, np.inf), 256)
    if positive:
        y = np.where(y > 0, np.maximum(y, 2.0 ** -9), y)
    a = np.abs(y)
    step = 2.0 ** (np.maximum(np.frexp(a)[1] - 1, -6) - 3)
    uu = np.zeros(nb * 256)
    uu[:n] = u
    pick = a / step + uu
    want = np.floor(pick) * step
    err = np.zeros(nb * 256)
    err[:n] = 4 * U * size
    err = err / np.repeat(np.where(top > 0, top / 448, np.inf), 256) / step + 2.0 ** -14
    border = np.abs(pick - np.round(pick)) <= err
    values = np.array([k * 2.0 ** -9 for k in range(8)] + [(8 + k) * 2.0 ** (e - 10) for e in range(1, 16) for k in range(8)][:-1])
    place = np.searchsorted(values, np.abs(code))
    beside = np.abs(place - np.searchsorted(values, want)) <= 1
    got = np.abs(code)
    assert np.all(values[place] == got) and np.all((got == want) | (border & beside)) and np.all(np.sign(code) == np.sign(y) * (got > 0))
    assert np.all(code[n:] == 0)


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 3])
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_moments_in_8_bits(sizes, K, gtype):
    p, g = _tensors(sizes, K, gtype, 4)
    if sizes[0] == 5000:
        g[0][:, 300:900] = 0        # a whole block and parts of two without gradients
    copies = [torch.zeros_like(x, dtype=torch.bfloat16) for x in p]
    opt = qsr.AdamW(p, g, states="fp8", copies=copies, weight_decay=0.1, beta1=B1, beta2=B2, eps=EPS, seed=99)
    for t in range(3):
        before, old = [x.clone() for x in p], [opt.moments(i) for i in range(len(p))]
        opt.step(1e-2, t)
        first = 0
        for i, n in enumerate(sizes):
            th, m, v, upd = _step64(before[i], g[i], old[i][0].double(), old[i][1].double(), 1e-2, t, 0.1)
            assert (p[i].double() - th).abs().le(3 * U * th.abs() + 60 * U * upd.abs() + 1e-12).all()
            assert torch.equal(copies[i], p[i].to(torch.bfloat16))
            if i in (0, 1, len(sizes) - 1):
                for k in range(K):
                    um, uv = _fractions(99, t, k, first, n)
                    c = lambda q: q[i][k].double().cpu().numpy()  # noqa: E731
                    size = (old[i][0][k].double().abs() + g[i][k].double().abs()).cpu().numpy()
                    r = v[k].sqrt().cpu().numpy()
                    _check_codes(c(opt.m), c(opt.m_scale), m[k].cpu().numpy(), size, um, False)
                    _check_codes(c(opt.v), c(opt.v_scale), r, r, uv, True)
            first += -(-n // 256) * 256


def test_moments_in_8_bits_follow_their_means():
    """Stochastic rounding: 400 steps of a constant gradient on 65536 elements bring the mean of the roots to where 32 bits are, within
    five standard errors of a random walk of half a code's step (2^-4 of the value at most), though no single step moves a code."""
    n = 65536
    g = [torch.full((1, n), 1e-3, device="cuda")]
    g[0][0, ::256] = 3e-3           # the block's largest: the others' codes are not at the end of the range
    opts = [qsr.AdamW([torch.zeros(1, n, device="cuda")], g, states=s, beta1=B1, beta2=B2, eps=EPS) for s in ("f32", "fp8")]
    for t in range(400):
        for o in opts:
            o.step(1e-3, t)
    (m, v), (m8, v8) = (o.moments(0) for o in opts)
    sel = torch.arange(n) % 256 != 0
    r, r8 = v[0, sel].sqrt().mean(), v8[0, sel].sqrt().mean()
    # the rounding feeds back into v: the mean of the roots is within a hundredth
    assert abs(float(r8 / r) - 1) < 0.01 and abs(float(m8[0, sel].mean() / m[0, sel].mean()) - 1) < 0.01


@pytest.mark.parametrize("states", ["f32", "fp8"])
def test_gradients_that_are_not_finite(states):
    """They spoil their own element and no other."""
    p, g = _tensors([1000], 1, torch.float32, 5)
    q = [p[0].clone()]
    bad = [17, 300, 999]
    clean = qsr.AdamW(q, [torch.where(torch.isin(torch.arange(1000, device="cuda"), torch.tensor(bad, device="cuda")), 0.0, g[0])],
                      states=states, beta1=B1, beta2=B2, eps=EPS)
    g[0][0, 17], g[0][0, 300], g[0][0, 999] = float("nan"), float("inf"), -float("inf")
    opt = qsr.AdamW(p, g, states=states, beta1=B1, beta2=B2, eps=EPS)
    for t in range(2):
        opt.step(1e-2, t)
        clean.step(1e-2, t)
    keep = ~torch.isin(torch.arange(1000), torch.tensor(bad)).cuda()
    assert p[0][0, bad].isnan().all() and torch.equal(p[0][:, keep], q[0][:, keep])
    m, _ = opt.moments(0)
    assert (~m[0, bad].isfinite()).all() and torch.equal(m[:, keep], clean.moments(0)[0][:, keep])


def test_rows_apart_other_gradients_and_streams():
    """Tensors as rows of one [K][P] buffer at odd places, gradients exchanged for others, moments handed on, another stream."""
    K, sizes, at = 3, [257, 1000, 33], [1, 301, 1400]
    buf = {k: torch.randn(K, 1501, generator=torch.Generator().manual_seed(i)).cuda() for i, k in enumerate("pgh")}
    views = lambda b: [b[:, o:o + n] for o, n in zip(at, sizes)]  # noqa: E731
    for states in ("f32", "fp8"):
        outside = buf["p"].clone()
        p = views(buf["p"])
        ref_p, ref_g, ref_h = ([x.clone() for x in views(buf[k])] for k in "pgh")
        opt = qsr.AdamW(p, views(buf["g"]), states=states, seed=3)
        ref = qsr.AdamW(ref_p, ref_g, states=states, seed=3)
        opt.step(1e-2, 0)
        ref.step(1e-2, 0)
        opt.set_grads(views(buf["h"]))
        ref.set_grads(ref_h)
        names = ("m", "v", "m_scale", "v_scale") if states == "fp8" else ("m", "v")
        more = qsr.AdamW(ref_p, ref_h, states=states, seed=3, moments={k: getattr(ref, k) for k in names})
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        opt.step(2e-2, 1, stream=side.cuda_stream)
        side.synchronize()
        more.step(2e-2, 1)
        for i in range(3):
            assert torch.equal(p[i], ref_p[i])
            assert all(torch.equal(a, b) for a, b in zip(opt.moments(i), more.moments(i)))
        mask = torch.ones(1501, dtype=torch.bool)
        for o, n in zip(at, sizes):
            mask[o:o + n] = False
        assert torch.equal(buf["p"][:, mask.cuda()], outside[:, mask.cuda()])


def test_other_gradients_for_many_tensors():
    """More tensors than one launch of addresses holds."""
    p, g = _tensors([3 + i % 5 for i in range(700)], 2, torch.bfloat16, 8)
    q, h = [x.clone() for x in p], [x.flip(1).contiguous() for x in g]
    a, b = qsr.AdamW(p, g), qsr.AdamW(q, h)
    a.set_grads(h)
    a.step(1e-2, 0)
    b.step(1e-2, 0)
    assert all(torch.equal(x, y) for x, y in zip(p, q))


def test_recorded_and_replayed():
    p, g = _tensors([5000, 70000, 3], 2, torch.float32, 9)
    q, h = [x.clone() for x in p], [x.clone() for x in g]
    a, b = (qsr.AdamW(x, y, states="fp8", clip_norm=0.5) for x, y in ((p, g), (q, h)))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a.step(1e-2, 4)
    for _ in range(3):
        graph.replay()
        b.step(1e-2, 4)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(p, q))
        assert all(torch.equal(a.m[i].view(torch.uint8), b.m[i].view(torch.uint8)) for i in range(3))
        torch.randn(1000, device="cuda").sum().item()


def test_workers_alone_and_together():
    """A worker's fp32 step does not depend on the others."""
    p, g = _tensors([700, 5], 4, torch.float32, 6)
    q, h = [x[2:3].clone() for x in p], [x[2:3].clone() for x in g]
    a, b = qsr.AdamW(p, g, clip_norm=0.01), qsr.AdamW(q, h, clip_norm=0.01)
    a.step(1e-2, 0)
    b.step(1e-2, 0)
    assert all(torch.equal(x[2:3], y) for x, y in zip(p, q))


def test_offsets_beyond_32_bits():
    """A tensor of more than 2^32 bytes a kind for two workers, its last elements."""
    n = (1 << 30) + 777
    p, g = torch.zeros(2, n, device="cuda"), torch.zeros(2, n, dtype=torch.bfloat16, device="cuda")
    p[:, -5:], g[:, -5:] = 1.0, 0.5
    opt = qsr.AdamW([p], [g], states="fp8", beta1=B1, beta2=B2, eps=EPS)
    opt.step(0.125, 0)
    assert torch.allclose(p[:, -5:], torch.full((2, 5), 0.875, device="cuda"), rtol=1e-6) and p[:, :-5].count_nonzero() == 0
    assert opt.m[0][:, n - 5:n].float().eq(448).all() and opt.m[0][:, :n - 5].view(torch.uint8).count_nonzero() == 0


def test_refusals():
    p, g = _tensors([10, 20], 2, torch.float32, 7)
    for bad in (dict(beta2=1.0), dict(eps=0.0), dict(clip_norm=-1.0), dict(weight_decay=-0.1), dict(weight_decay=[0.1]), dict(states="int8"),
                dict(copies=p), dict(moments={"m": p, "v": p[:1]})):
        with pytest.raises(ValueError):
            qsr.AdamW(p, g, **bad)
    for args in (([], []), (p, g[:1]), ([p[0].double()], g[:1]), (p, [g[0], g[1].bfloat16()]), (p, [g[0], g[1][:, :5]]),
                 ([p[0].t()], [g[0].t()]), ([p[0][:1].expand(2, 10)], g[:1])):
        with pytest.raises(ValueError):
            qsr.AdamW(*args)
    opt = qsr.AdamW(p, g)
    with pytest.raises(ValueError):
        opt.set_grads([g[0], g[1].bfloat16()])
    for eta, t in ((float("nan"), 0), (-1.0, 0), (1e-3, -1)):
        with pytest.raises(qsr.QSRError) as e:
            opt.step(eta, t)
        assert e.value.code == -1


def test_step_numbers_have_an_end():
    p, g = _tensors([10], 1, torch.float32, 10)
    opt = qsr.AdamW(p, g)
    with pytest.raises(qsr.QSRError) as e:
        opt.step(1e-3, 2 ** 63 - 1)
    assert e.value.code == -1
    opt.step(1e-3, 2 ** 63 - 2)
    assert p[0].isfinite().all()


@pytest.mark.parametrize("blocks", [1023, 1024, 1025, 2048, 2600])
def test_every_block_is_taken_once(blocks):
    """Lists around whole groups of trips, with 8-bit moments: after two steps of a gradient that is the same everywhere, from the same
    parameters, every element is where the others are but for the second step's rounded moments (a code is off by 2^-3 at most), and
    every block has its scale."""
    n = blocks * 256 - 100
    p, g = [torch.ones(2, n, device="cuda"), torch.ones(2, 300, device="cuda")], [torch.full((2, n), 1e-2, device="cuda"),
                                                                                 torch.full((2, 300), 1e-2, device="cuda")]
    opt = qsr.AdamW(p, g, states="fp8", beta1=B1, beta2=B2, eps=EPS)
    opt.step(1e-3, 0)
    for x in p:         # m and r are still exact where they are used: a step of eta
        assert (x.double() - (1 - 1e-3)).abs().max() <= 2 ** -24 * 2
    opt.step(1e-3, 1)
    for i, x in enumerate(p):
        assert (x.double() - (1 - 2e-3)).abs().max() <= 1e-3 * 2 ** -2
        for s, want in ((opt.m_scale[i], 1.9e-3), (opt.v_scale[i], 1e-2 * (1 - B2 ** 2) ** 0.5)):
            assert ((s.double() * 448 - want).abs() <= want * 2 ** -3).all()
