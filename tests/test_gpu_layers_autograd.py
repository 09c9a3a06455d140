"""Layer norm, the embedding and the gated recurrence beside torch's automatic differentiation: they record no graph."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu


def _arguments():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    x, w, b, res, dy = r(4, 32), r(32), r(32), r(4, 32), r(4, 32)
    tok, table = torch.tensor([1, 5, 31, -1]).cuda(), r(40, 32)
    u, f, st = r(2, 20, 8), r(2, 20, 8), r(2, 8)
    n, s = qsr.layernorm(x, w, b, residual=res), qsr.gated_scan(u, f, initial=st, keep=True)
    calls = {
        "layernorm": (lambda a: qsr.layernorm(a["x"], a["w"], a["b"], residual=a["res"], sum_out=a["out"]),
                      dict(x=x, w=w, b=b, res=res, out=torch.empty_like(x))),
        "layernorm_backward": (lambda a: qsr.layernorm_backward(a["dy"], a["s"], a["w"], a["mean"], a["rstd"], a["res"]),
                               dict(dy=dy, s=n.sum, w=w, mean=n.mean, rstd=n.rstd, res=res)),
        "embedding": (lambda a: qsr.embedding(tok, a["table"]), dict(table=table)),
        "embedding_backward": (lambda a: qsr.embedding_backward(a["dy"], tok, table, out=a["out"]), dict(dy=dy, out=torch.empty_like(table))),
        "gated_scan": (lambda a: qsr.gated_scan(a["u"], a["f"], initial=a["st"], keep=True, state_out=a["out"]),
                       dict(u=u, f=f, st=st, out=torch.empty_like(st))),
        "gated_scan_backward": (lambda a: qsr.gated_scan_backward(a["dh"], a["u"], a["f"], a["states"], last_grad=a["dl"]),
                                dict(dh=r(2, 20, 8), u=u, f=f, states=s.states, dl=r(2, 8))),
    }
    return [(call, args, name, key) for name, (call, args) in calls.items() for key in args]


def test_tensors_that_want_gradients_are_refused():
    for call, args, name, key in _arguments():
        want = call({k: v.clone() for k, v in args.items()})
        mine = {k: v.clone().requires_grad_(k == key) for k, v in args.items()}
        with pytest.raises(ValueError, match="gradient"):
            call(mine)
        with torch.no_grad():
            got = call(mine)
        for a, b in zip(*((r if isinstance(r, tuple) else (r,)) for r in (want, got))):
            assert (a is None and b is None) or torch.equal(a, b), (name, key)
        call({k: v.detach() for k, v in mine.items()})


def test_a_table_that_wants_gradients_gives_its_shape():
    """The gradient's call takes nothing of the table but shape, type and place."""
    table, tok = torch.zeros(5, 8, device="cuda", requires_grad=True), torch.tensor([1, 1, 4], device="cuda")
    got = qsr.embedding_backward(torch.ones(3, 8, device="cuda"), tok, table)
    assert got[:, 0].tolist() == [0, 2, 0, 0, 1] and not got.requires_grad


def test_results_in_place_are_new_versions():
    """What is written in place counts as written: a graph that has kept the tensor finds out in its backward pass."""
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn(4, 32, generator=g).cuda(), torch.ones(32, device="cuda")
    tok, u = torch.tensor([0, 3, 3, 1], device="cuda"), torch.randn(4, 6, 32, generator=g).cuda()
    writes = (lambda out: qsr.layernorm(x, w, residual=x, sum_out=out), lambda out: qsr.embedding_backward(x, tok, out, out=out),
              lambda out: qsr.embedding_backward(x, tok, out, out=out, accumulate=True), lambda out: qsr.gated_scan(u, u, initial=out, state_out=out))
    for write in writes:
        out = torch.randn(4, 32, device="cuda")
        a = torch.ones(4, 32, device="cuda", requires_grad=True)
        kept, before = (a * out).sum(), out._version
        write(out)
        assert out._version > before
        with pytest.raises(RuntimeError, match="inplace"):
            kept.backward()


def test_tensors_of_inference_have_no_versions():
    with torch.inference_mode():
        x, w, st = torch.randn(4, 3, 32, device="cuda"), torch.ones(32, device="cuda"), torch.zeros(4, 32, device="cuda")
        f = qsr.layernorm(x, w, w, residual=x, sum_out=x)
        s = qsr.gated_scan(x, x, initial=st, state_out=st)
        assert f.sum is x and s.last is st
        assert qsr.embedding(torch.tensor([2], device="cuda"), w[:, None]).shape == (1, 1)


def test_two_streams_at_once():
    """Calls on two streams have workspaces of their own: the results of each alone, many times over."""
    g = torch.Generator().manual_seed(3)
    dy, tok, table = torch.randn(6000, 24, generator=g).cuda(), torch.randint(0, 300, (6000,), generator=g).cuda(), torch.empty(300, 24, device="cuda")
    u, f = torch.randn(1, 5000, 40, generator=g).cuda(), torch.randn(1, 5000, 40, generator=g).cuda()
    x, w = torch.randn(700, 96, generator=g).cuda(), torch.ones(96, device="cuda")

    def run(stream=None):
        s = qsr.gated_scan(u, f, keep=True, stream=stream)
        n = qsr.layernorm(x, w, w, stream=stream)
        return (qsr.embedding_backward(dy, tok, table, stream=stream), s.h, *qsr.gated_scan_backward(u, u, f, s.states, stream=stream),
                *qsr.layernorm_backward(x, x, w, n.mean, n.rstd, stream=stream))
    want = run()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(8):
        for s in sides:
            got.append(run(s.cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for r in got for p, q in zip(r, want))


def test_memory_from_elsewhere():
    """Arguments whose memory is not from torch's allocator (a capsule of another library's): results are torch's all the same."""
    x, w, tok = torch.randn(5, 3, 32, device="cuda"), torch.ones(32, device="cuda"), torch.tensor([1, 0, 4], device="cuda")
    other = torch.from_dlpack(torch.utils.dlpack.to_dlpack(x))
    for call in (lambda t: qsr.layernorm(t, w, w, residual=t), lambda t: qsr.gated_scan(t, t, keep=True), lambda t: (qsr.embedding(tok, t[0]),),
                 lambda t: (qsr.embedding_backward(t[0], tok, t[:, 0]),), lambda t: qsr.rmsnorm(t, w)):
        got = [v for v in call(other) if v is not None]
        assert all(torch.equal(a, b) and a.device == x.device for a, b in zip(got, [v for v in call(x) if v is not None]))
        assert all(v.is_contiguous() and not v.requires_grad for v in got)
