"""The gated linear recurrence and its gradients against the formulas in 64 bits, step by step.

Tolerances.  U = 2^-24 and B = 2^-8 are the unit roundoffs of fp32 and bf16.  A gate's a and 1 - a are off by G relatively: the exponential by 3 U,
its sum with one, the reciprocal and the product by 5 more at most; from bf16 gates the exponent's product has 1.3 |f| U beside it.  State t is a sum of terms (w_j x_j, or the initial state) times the gates of the steps since, in whatever order the steps are joined: each factor brings
G and a rounding, each join (one in sixteen steps) and each addition another, so that it is off by (G + 3 U) N_t + 6 U M_t at most with
M_t = a_t M_{t-1} + |w_t x_t|, the sum of the terms' sizes, and N_t = a_t (N_{t-1} + M_{t-1}) + |w_t x_t|, where each counts as often as it has
factors.  The gradients g_t are such sums from the other end.  dx = w g and df = g a c (h - x) have a rounding or G for each factor on
top, and the error of h; what is stored in bf16 its own rounding."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _half(dt):
    return 0.0 if dt == torch.float32 else B


def _data(B_, T, d, dt, seed, full):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    s = dict(x=r(B_, T, d).to(dt), gate=(r(B_, T, d) * 2 + 4 * torch.rand(d, generator=g)).to(dt), dh=r(B_, T, d).to(dt))
    if full:
        s.update(initial=r(B_, d), reset=torch.rand(B_, T, generator=g) < 0.02, dlast=r(B_, d),
                 lengths=torch.tensor([[T, 0, 1, T // 2, T + 5, -3][i % 6] for i in range(B_)]))
    return {k: v.cuda() for k, v in s.items()}


def _exact(s, plain):
    """h, last, dx, dgate, dinitial in 64 bits, each with its bound."""
    x, f, dh = (s[k].double() for k in ("x", "gate", "dh"))
    B_, T, d = x.shape
    zero = torch.zeros(B_, d, dtype=torch.float64, device=x.device)
    G = (8 if s["x"].dtype == torch.float32 else 2 * float(f.abs().max()) + 8 if f.numel() else 0) * U
    a, c = torch.sigmoid(f), torch.sigmoid(-f)
    w = torch.ones_like(c) if plain else c
    end = s["lengths"].clamp(0, T) if "lengths" in s else torch.full((B_,), T, device=x.device)
    live = [(end > t)[:, None] for t in range(T)]
    cut = [s["reset"][:, t, None] if "reset" in s else torch.zeros(B_, 1, dtype=torch.bool, device=x.device) for t in range(T)]
    bound = lambda N, M: (G + 3 * U) * N + 6 * U * M  # noqa: E731
    h, M, N = s["initial"].double() if "initial" in s else zero, None, zero
    M = h.abs()
    out = {k: torch.zeros_like(x) for k in ("h", "h_", "dx", "dx_", "dgate", "dgate_", "p", "p_")}
    for t in range(T):
        h0, M0, N0 = (torch.where(cut[t], zero, v) for v in (h, M, N))
        out["p"][:, t], out["p_"][:, t] = h0, bound(N0, M0)
        b = w[:, t] * x[:, t]
        h1, M1, N1 = a[:, t] * h0 + b, a[:, t] * M0 + b.abs(), a[:, t] * (N0 + M0) + b.abs()
        h, M, N = (torch.where(live[t], new, old) for new, old in ((h1, h), (M1, M), (N1, N)))
        out["h"][:, t], out["h_"][:, t] = torch.where(live[t], h1, zero), torch.where(live[t], bound(N1, M1), zero)
    last, last_ = h, bound(N, M)
    e = s["dlast"].double() if "dlast" in s else zero
    M, N = e.abs(), zero
    for t in range(T - 1, -1, -1):
        g, gM = e + dh[:, t], M + dh[:, t].abs()
        g_ = bound(N + gM, gM)
        p = out["p"][:, t] - (0 if plain else x[:, t])
        p_ = out["p_"][:, t] + U * p.abs()
        ac = a[:, t] * c[:, t]
        vals = dict(dx=w[:, t] * g, dx_=w[:, t] * (g_ + (G + 2 * U) * g.abs()), dgate=g * ac * p,
                    dgate_=ac * (g_ * p.abs() + (g.abs() + g_) * p_) + (2 * G + 6 * U) * (g * ac * p).abs())
        for k, v in vals.items():
            out[k][:, t] = torch.where(live[t], v, zero)
        e1, M1, N1 = a[:, t] * g, a[:, t] * gM, a[:, t] * (N + gM)
        e, M, N = (torch.where(live[t], torch.where(cut[t], zero, new), old) for new, old in ((e1, e), (M1, M), (N1, N)))
    return out, (last, last_), (e, bound(N, M))


def _near(got, want, room, what):
    half = _half(got.dtype)
    ok = (got.double() - want).abs().le(room + half * (want.abs() + room) + (2.0 ** -133 if half else 2.0 ** -126))
    assert ok.all(), (what, got[~ok][:4], want[~ok][:4], room[~ok][:4])


def _marks(s, plain):
    return dict(reset=s.get("reset"), lengths=s.get("lengths"), input="plain" if plain else "complement")


SIZES = [(1, 1, 1), (2, 1, 5), (5, 1, 200), (1, 2, 3), (6, 16, 64), (2, 17, 130), (1, 127, 7), (7, 128, 128), (1, 129, 65), (6, 300, 33), (1, 1100, 9),
         (6, 1500, 40), (1, 3001, 129), (130, 300, 30), (200, 270, 3), (520, 20, 5)]


@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B_,T,d", SIZES)
def test_both_passes(B_, T, d, dt, plain, full):
    s = _data(B_, T, d, DT[dt], 1, full)
    f = qsr.gated_scan(s["x"], s["gate"], initial=s.get("initial"), keep=True, **_marks(s, plain))
    want, last, first = _exact(s, plain)
    assert f.h.dtype == DT[dt] and f.last.shape == (B_, d) and f.states.shape == (B_, -(-T // 16), d)
    _near(f.h, want["h"], want["h_"], "h")
    _near(f.last, *last, "last")
    none = qsr.gated_scan(s["x"], s["gate"], initial=s.get("initial"), **_marks(s, plain))
    assert none.states is None and torch.equal(none.h, f.h) and torch.equal(none.last, f.last)
    dx, dgate, dinitial = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, last_grad=s.get("dlast"), **_marks(s, plain))
    assert dx.dtype == dgate.dtype == DT[dt] and dinitial.dtype == torch.float32
    _near(dx, want["dx"], want["dx_"], "dx")
    _near(dgate, want["dgate"], want["dgate_"], "dgate")
    _near(dinitial, *first, "dinitial")


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("T", [5, 40])
def test_gradient_against_differences(T, plain):
    """Central differences, in 64 bits, of sum(h dh) + sum(last dlast): truncation h^2 = 1e-10, cancellation 1e-16 / h = 1e-11, both
    times sums of some hundred terms of size one; the gradient itself is fp32."""
    s = _data(6, T, 2, torch.float32, 2, True)
    s["reset"][0, T // 2] = True
    f = qsr.gated_scan(s["x"], s["gate"], initial=s["initial"], keep=True, **_marks(s, plain))
    got = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, last_grad=s["dlast"], **_marks(s, plain))
    cpu = {k: v.cpu() for k, v in s.items()}

    def value(x, gate, initial):
        a = torch.sigmoid(gate)
        h, total = initial, 0.0
        for t in range(T):
            live = (cpu["lengths"] > t)[:, None]
            new = a[:, t] * torch.where(cpu["reset"][:, t, None], torch.zeros_like(h), h) + (1 if plain else 1 - a[:, t]) * x[:, t]
            total = total + float((torch.where(live, new, torch.zeros_like(new)) * cpu["dh"][:, t]).sum())
            h = torch.where(live, new, h)
        return total + float((h * cpu["dlast"]).sum())
    for i, (name, grad) in enumerate(zip(("x", "gate", "initial"), got)):
        scale = float(grad.abs().max())
        for j in range(0, grad.numel(), 3):
            two = []
            for sign in (1e-5, -1e-5):
                args = [cpu[k].double().clone() for k in ("x", "gate", "initial")]
                args[i].view(-1)[j] += sign
                two.append(value(*args))
            assert abs((two[0] - two[1]) / 2e-5 - float(grad.view(-1)[j])) <= 1e-5 * (1 + scale), name


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_one_step_at_a_time(dt):
    """A text goes on from where it was, in pieces down to single tokens whose states are updated in place: as all of it at once."""
    s = _data(3, 150, 70, DT[dt], 3, False)
    want, last, _ = _exact(s, False)
    state, got, at = torch.zeros(3, 70, device="cuda"), [], 0
    for n in (100, 17, 16, 5) + (1,) * 12:
        f = qsr.gated_scan(s["x"][:, at:at + n], s["gate"][:, at:at + n], initial=state, state_out=state)
        assert f.last is state
        got.append(f.h)
        at += n
    _near(torch.cat(got, 1), want["h"], want["h_"], "h")
    _near(state, *last, "last")


def test_states_in_place_of_many_parts():
    """One sequence on many workgroups, the last of which writes what the first one reads."""
    s = _data(1, 6000, 70, torch.bfloat16, 4, False)
    for d in (70, 69, 1):
        x, gate = s["x"][..., :d], s["gate"][..., :d]
        state = torch.randn(1, d, generator=torch.Generator().manual_seed(5)).cuda()
        f = qsr.gated_scan(x, gate, initial=state)
        for _ in range(3):
            again = state.clone()
            g = qsr.gated_scan(x, gate, initial=again, state_out=again)
            assert torch.equal(g.h, f.h) and torch.equal(again, f.last)


@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("B_,T,d", [(100, 16, 255), (100, 20, 253), (100, 64, 255), (90, 140, 130), (150, 290, 101), (300, 131, 251), (7, 2500, 700),
                                    (7, 2600, 641)])
def test_two_channels_of_a_lane(B_, T, d, plain, full):
    """Enough workgroups for them: one to sixteen wavefronts, parts; even and odd rows, in tensors of their own and inside others."""
    s = _data(B_, T, d, torch.bfloat16, 18, full)
    marks = _marks(s, plain)
    f = qsr.gated_scan(s["x"], s["gate"], initial=s.get("initial"), keep=True, **marks)
    back = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, last_grad=s.get("dlast"), **marks)
    want, last, first = _exact(s, plain)
    _near(f.h, want["h"], want["h_"], "h")
    _near(f.last, *last, "last")
    _near(back[0], want["dx"], want["dx_"], "dx")
    _near(back[1], want["dgate"], want["dgate_"], "dgate")
    _near(back[2], *first, "dinitial")
    both = torch.full((T, B_, 2 * d + 3), float("nan"), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    x, gate = both[..., 1:1 + d], both[..., 2 + d:2 + 2 * d]
    x.copy_(s["x"]), gate.copy_(s["gate"])
    state = s["initial"].clone() if full else None
    g = qsr.gated_scan(x, gate, initial=state, keep=True, state_out=state, **marks)
    again = qsr.gated_scan_backward(s["dh"], x, gate, g.states, last_grad=s.get("dlast"), **marks)
    assert all(torch.equal(p, q) for p, q in zip(f + tuple(back), g + tuple(again)))


@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B_,T,d", [(6, 18, 5), (2, 31, 64), (3, 32, 131), (6, 33, 3), (70, 47, 65), (2, 64, 300), (5, 65, 70), (6, 128, 20)])
def test_short_sequences(B_, T, d, dt, full):
    """Two and four wavefronts to a workgroup, with and without steps for all of them."""
    for plain in (False, True):
        test_both_passes(B_, T, d, dt, plain, full)


@pytest.mark.parametrize("dt,d,full", [("bf16", 3, True), ("f32", 65, False)])
def test_more_parts_than_wavefronts(dt, d, full):
    """157 parts: each wavefront joins the maps of twenty of them, of the last one fewer."""
    s = _data(1, 20001, d, DT[dt], 17, full)
    f = qsr.gated_scan(s["x"], s["gate"], initial=s.get("initial"), keep=True, **_marks(s, False))
    want, last, first = _exact(s, False)
    _near(f.h, want["h"], want["h_"], "h")
    _near(f.last, *last, "last")
    dx, dgate, dinitial = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, last_grad=s.get("dlast"), **_marks(s, False))
    _near(dx, want["dx"], want["dx_"], "dx")
    _near(dgate, want["dgate"], want["dgate_"], "dgate")
    _near(dinitial, *first, "dinitial")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T", [9, 200, 3000])
def test_pieces_of_a_sequence_backward(T, dt):
    """Gradients through the state between two calls are those of one call."""
    s = _data(2, T, 40, DT[dt], 6, False)
    s["dlast"] = torch.randn(2, 40, generator=torch.Generator().manual_seed(7)).cuda()
    want, _, first = _exact(s, False)
    m = T // 3
    a, b = {k: v[:, :m] for k, v in s.items() if v.dim() == 3}, {k: v[:, m:] for k, v in s.items() if v.dim() == 3}
    fa = qsr.gated_scan(a["x"], a["gate"], keep=True)
    fb = qsr.gated_scan(b["x"], b["gate"], initial=fa.last, keep=True)
    gb = qsr.gated_scan_backward(b["dh"], b["x"], b["gate"], fb.states, last_grad=s["dlast"])
    ga = qsr.gated_scan_backward(a["dh"], a["x"], a["gate"], fa.states, last_grad=gb[2])
    _near(torch.cat([ga[0], gb[0]], 1), want["dx"], want["dx_"], "dx")
    _near(torch.cat([ga[1], gb[1]], 1), want["dgate"], want["dgate_"], "dgate")
    _near(ga[2], *first, "dinitial")


@pytest.mark.parametrize("T", [13, 100, 4000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_documents_are_apart(dt, T):
    """What is not finite before a reset, or behind a sequence's end, is not seen on the other side, in either direction."""
    s = _data(2, T, 20, DT[dt], 8, False)
    cut = 2 * T // 3
    s["reset"] = torch.zeros(2, T, dtype=torch.bool, device="cuda")
    s["reset"][:, cut] = True
    s["lengths"] = torch.tensor([T - 2, T - 2]).cuda()
    marks = _marks(s, False)
    f = qsr.gated_scan(s["x"], s["gate"], keep=True, **marks)
    back = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, **marks)
    for bad in (float("nan"), float("inf")):
        x, gate, dh = s["x"].clone(), s["gate"].clone(), s["dh"].clone()
        x[0, T // 3:cut] = bad
        gate[1, T // 3:cut] = float("nan")
        x[:, T - 2:] = gate[:, T - 2:] = dh[:, T - 2:] = bad
        g = qsr.gated_scan(x, gate, initial=torch.full((2, 20), bad, device="cuda"), keep=True, **marks)
        assert torch.equal(g.h[:, cut:], f.h[:, cut:]) and torch.equal(g.last, f.last) and not g.h[:, cut - 1].isfinite().any()
        dx, dgate, _ = qsr.gated_scan_backward(dh, x, gate, g.states, **marks)
        assert torch.equal(dx[:, cut:], back[0][:, cut:])
        assert torch.equal(dgate[:, cut:], back[1][:, cut:])
        # and from the later document into the earlier one
        x, dh = s["x"].clone(), s["dh"].clone()
        dh[:, cut:] = bad
        x[:, cut:] = bad
        g = qsr.gated_scan(x, s["gate"], keep=True, **marks)
        dx, dgate, dinitial = qsr.gated_scan_backward(dh, x, s["gate"], g.states, last_grad=torch.full((2, 20), bad, device="cuda"), **marks)
        assert torch.equal(dx[:, :cut], back[0][:, :cut]) and torch.equal(dgate[:, :cut], back[1][:, :cut]) and torch.equal(dinitial, back[2])


@pytest.mark.parametrize("T", [3, 40])
def test_gates_at_their_ends(T):
    """Infinite gates keep or replace the state, exactly; huge ones are the same without an overflow."""
    x = torch.arange(1.0, T + 1, device="cuda")[None, :, None].expand(1, T, 6).contiguous()
    for big in (float("inf"), 3e38, 200.0):
        gate = torch.full((1, T, 6), big, device="cuda")
        gate[:, 1] = -big
        f = qsr.gated_scan(x, gate, initial=torch.full((1, 6), 9.0, device="cuda"), keep=True)
        assert f.h[0, 0].eq(9).all() and f.h[0, 1:].eq(2).all()
        dx, dgate, dinitial = qsr.gated_scan_backward(torch.ones_like(x), x, gate, f.states)
        assert dx[0, 0].eq(0).all() and dx[0, 1].eq(T - 1).all() and dx[0, 2:].eq(0).all() and dgate.eq(0).all() and dinitial.eq(1).all()


def test_strides_and_places():
    """Two halves of one product's output, time before batch, channels that start at any element, and another stream: the same."""
    for dt in DT.values():
        for T, d in ((1, 33), (12, 33), (300, 33), (2000, 10)):
            s = _data(3, T, d, dt, 9, True)
            marks = _marks(s, False)
            f = qsr.gated_scan(s["x"], s["gate"], initial=s["initial"], keep=True, **marks)
            back = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, last_grad=s["dlast"], **marks)
            both = torch.full((3, T, 2 * d + 3), float("nan"), dtype=dt, device="cuda")
            turned = [torch.full((T, 3, d), float("nan"), dtype=dt, device="cuda").transpose(0, 1) for _ in range(3)]
            for x, gate, dh in ((both[..., 1:1 + d], both[..., 2 + d:2 + 2 * d], s["dh"]), turned):
                x.copy_(s["x"]), gate.copy_(s["gate"]), dh.copy_(s["dh"])
                g = qsr.gated_scan(x, gate, initial=s["initial"], keep=True, **marks)
                assert all(torch.equal(p, q) for p, q in zip(f, g))
                again = qsr.gated_scan_backward(dh, x, gate, g.states, last_grad=s["dlast"], **marks)
                assert all(torch.equal(p, q) for p, q in zip(back, again))
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            g = qsr.gated_scan(s["x"], s["gate"], initial=s["initial"], keep=True, stream=side.cuda_stream, **marks)
            again = qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], g.states, last_grad=s["dlast"], stream=side.cuda_stream, **marks)
            side.synchronize()
            assert torch.equal(g.h, f.h) and all(torch.equal(p, q) for p, q in zip(back, again))


def test_shapes():
    """No sequences, no steps, no dimension for sequences, several."""
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    f = qsr.gated_scan(z(0, 5, 4), z(0, 5, 4), keep=True)
    assert f.h.shape == (0, 5, 4) and f.last.shape == (0, 4) and f.states.shape == (0, 1, 4)
    assert qsr.gated_scan_backward(z(0, 5, 4), z(0, 5, 4), z(0, 5, 4), f.states)[2].shape == (0, 4)
    start = torch.ones(2, 4, device="cuda")
    f = qsr.gated_scan(z(2, 0, 4), z(2, 0, 4), initial=start, keep=True)
    assert f.h.shape == (2, 0, 4) and torch.equal(f.last, start) and f.states.shape == (2, 0, 4)
    assert torch.equal(qsr.gated_scan_backward(z(2, 0, 4), z(2, 0, 4), z(2, 0, 4), f.states, last_grad=3 * start)[2], 3 * start)
    assert qsr.gated_scan(z(2, 0, 4), z(2, 0, 4)).last.eq(0).all()
    s = _data(6, 30, 8, torch.float32, 10, False)
    f = qsr.gated_scan(s["x"], s["gate"])
    g = qsr.gated_scan(s["x"].view(2, 3, 30, 8), s["gate"].view(2, 3, 30, 8))
    assert torch.equal(g.h.view(6, 30, 8), f.h) and g.last.shape == (2, 3, 8)
    g = qsr.gated_scan(s["x"][4], s["gate"][4], lengths=torch.tensor(30).cuda(), reset=torch.zeros(30, dtype=torch.bool, device="cuda"))
    assert torch.equal(g.h, f.h[4]) and g.last.shape == (8,)


@pytest.mark.parametrize("T", [1, 200, 4000])
def test_recorded_and_replayed(T):
    """Values, marks and lengths change between the replays."""
    s = _data(2, T, 24, torch.bfloat16, 11, True)
    def both():
        f = qsr.gated_scan(s["x"], s["gate"], initial=s["initial"], keep=True, **_marks(s, False))
        return (*f, *qsr.gated_scan_backward(s["dh"], s["x"], s["gate"], f.states, last_grad=s["dlast"], **_marks(s, False)))
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(3):
        for k, v in _data(2, T, 24, torch.bfloat16, 12 + i, True).items():
            s[k].copy_(v)
        s["lengths"].copy_(torch.tensor([T, T // 2 + i]))
        want = both()
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_refusals():
    x = torch.zeros(3, 20, 8, device="cuda")
    st, reset, n = torch.zeros(3, 8, device="cuda"), torch.zeros(3, 20, dtype=torch.bool, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    kept = torch.zeros(3, 2, 8, device="cuda")
    for call in (lambda: qsr.gated_scan(x.half(), x.half()), lambda: qsr.gated_scan(x, x.bfloat16()), lambda: qsr.gated_scan(x, x[:, :19]),
                 lambda: qsr.gated_scan(x[0, 0], x[0, 0]), lambda: qsr.gated_scan(x.transpose(1, 2), x.transpose(1, 2)), lambda: qsr.gated_scan(x, x.cpu()),
                 lambda: qsr.gated_scan(x, x, initial=st[:2]), lambda: qsr.gated_scan(x, x, initial=st.bfloat16()),
                 lambda: qsr.gated_scan(x, x, initial=torch.zeros(8, 3, device="cuda").t()), lambda: qsr.gated_scan(x, x, state_out=st.double()),
                 lambda: qsr.gated_scan(x, x, reset=reset[:, :19]), lambda: qsr.gated_scan(x, x, reset=reset.float()), lambda: qsr.gated_scan(x, x, lengths=n.int()),
                 lambda: qsr.gated_scan(x, x, lengths=n[:2]), lambda: qsr.gated_scan(x, x, lengths=n.cpu()),
                 lambda: qsr.gated_scan_backward(x[:, :19], x, x, kept), lambda: qsr.gated_scan_backward(x, x, x, kept[:, :1]),
                 lambda: qsr.gated_scan_backward(x, x, x, None), lambda: qsr.gated_scan_backward(x, x, x, kept, last_grad=st.bfloat16())):
        with pytest.raises(ValueError):
            call()
    for y in (x.expand(3, 20, 8)[:, :1].expand(3, 20, 8), x[:1].expand(3, 20, 8)):      # broadcast steps or sequences
        with pytest.raises(qsr.QSRError):
            qsr.gated_scan(y, x)
