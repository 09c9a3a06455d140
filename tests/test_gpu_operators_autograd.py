"""The operators beside torch's automatic differentiation: they record no graph."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu


def _arguments():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    x, w, res, dy = r(4, 32), r(32), r(4, 32), r(4, 32)
    tok = torch.tensor([1, 5, 31, -1]).cuda()
    f, t = qsr.rmsnorm(x, w, residual=res), qsr.token_logprobs(x, tok)
    calls = {
        "rmsnorm": (lambda a: qsr.rmsnorm(a["x"], a["w"], residual=a["res"], sum_out=a["out"]),
                    dict(x=x, w=w, res=res, out=torch.empty_like(x))),
        "rmsnorm_backward": (lambda a: qsr.rmsnorm_backward(a["dy"], a["s"], a["w"], a["rstd"], a["res"]),
                             dict(dy=dy, s=f.sum, w=w, rstd=f.rstd, res=res)),
        "token_logprobs": (lambda a: qsr.token_logprobs(a["x"], tok, top=3), dict(x=x)),
        "token_logprobs_backward": (lambda a: qsr.token_logprobs_backward(a["x"], tok, a["stats"], a["H"], a["da"], a["db"], out=a["out"]),
                                    dict(x=x, stats=t.stats, H=t.entropy, da=r(4), db=r(4), out=torch.empty_like(x))),
    }
    return [(call, args, name, key) for name, (call, args) in calls.items() for key in args]


def test_tensors_that_want_gradients_are_refused():
    """A result without a graph where a gradient is asked for would be a gradient lost in silence; without recording, and of
    detached tensors, the calls are what they were."""
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


def test_parameters_that_want_gradients_are_updated():
    """An optimizer's step on leaves, as torch's own make it."""
    p = [torch.ones(1, 40, device="cuda").requires_grad_(), torch.ones(1, 3, device="cuda").requires_grad_()]
    q = [x.detach().clone() for x in p]
    g = [torch.full_like(x, 0.5) for x in q]
    for params in (p, q):
        qsr.AdamW(params, g).step(1e-2, 0)
    assert all(torch.equal(a, b) and a.requires_grad for a, b in zip(p, q)) and float(q[0][0, 0].detach()) < 1


def test_results_in_place_are_new_versions():
    """What is written in place counts as written: a graph that has kept the tensor finds out in its backward pass."""
    g = torch.Generator().manual_seed(2)
    x, w, tok = torch.randn(4, 32, generator=g).cuda(), torch.ones(32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    t = qsr.token_logprobs(x, tok)

    def norm(out):
        qsr.rmsnorm(x, w, residual=x, sum_out=out)

    def logits(out):
        qsr.token_logprobs_backward(x, tok, t.stats, t.entropy, t.logp, out=out)
    for write in (norm, logits):
        for out in (torch.randn(4, 32, device="cuda"), torch.randn(4, 40, device="cuda")[:, 3:35]):
            a = torch.ones(4, 32, device="cuda", requires_grad=True)
            kept, before = (a * out).sum(), out._version
            write(out)
            assert out._version > before
            with pytest.raises(RuntimeError, match="inplace"):
                kept.backward()


@pytest.mark.parametrize("states", ["f32", "fp8"])
def test_steps_are_new_versions(states):
    """Parameters, copies and moments of a step, as tensors of their own or as views of one buffer; gradients are only read."""
    flat = torch.zeros(2, 60, device="cuda")
    for p in ([torch.zeros(2, 40, device="cuda"), torch.zeros(2, 3, device="cuda")], [flat[:, :40], flat[:, 44:47]]):
        grads, copies = [torch.ones_like(x) for x in p], [x.to(torch.bfloat16) for x in p]
        opt = qsr.AdamW(p, grads, states=states, copies=copies)
        written = p + copies + opt.m + opt.v + (opt.m_scale + opt.v_scale if states == "fp8" else [])
        for t in range(2):
            before, read = [x._version for x in written], [x._version for x in grads]
            a = torch.ones_like(p[1], requires_grad=True)
            kept = (a * p[1]).sum()
            opt.step(1e-2, t)
            assert all(x._version > v for x, v in zip(written, before)) and [x._version for x in grads] == read
            with pytest.raises(RuntimeError, match="inplace"):
                kept.backward()


def test_tensors_of_inference_have_no_versions():
    with torch.inference_mode():
        x, w, p = torch.randn(4, 32, device="cuda"), torch.ones(32, device="cuda"), torch.zeros(1, 5, device="cuda")
        f = qsr.rmsnorm(x, w, residual=x, sum_out=x)
        opt = qsr.AdamW([p], [torch.ones_like(p)])
        opt.step(1e-2, 0)
    opt.step(1e-2, 1)
    assert f.sum is x and bool(p.lt(0).all())
