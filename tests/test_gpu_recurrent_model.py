"""The example that runs the embedding, layer norm and the gated recurrence with the other operators: K workers train a recurrent model."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("local_recurrent_tokens", os.path.join(ROOT, "examples", "local_recurrent_tokens.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _value(p, tok, target, first):
    """The model's mean loss in 64 bits, for one worker."""
    def norm(x, g, b):
        v = x - x.mean(-1, keepdim=True)
        return v / (v.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * g + b
    x = p["E"][tok]
    v, f = (norm(x, p["g1"], p["b1"]) @ p["Wi"]).chunk(2, -1)
    a, h, hs = torch.sigmoid(f), torch.zeros_like(x[:, 0]), []
    for t in range(tok.shape[1]):
        h = a[:, t] * torch.where(first[:, t, None], torch.zeros_like(h), h) + (1 - a[:, t]) * v[:, t]
        hs.append(h)
    z = norm(x + torch.stack(hs, 1) @ p["Wo"], p["g2"], p["b2"]) @ p["Wv"]
    return torch.nn.functional.cross_entropy(z.flatten(0, 1), target.flatten(), ignore_index=-1)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2.0 ** -12), (torch.bfloat16, 0.07)])
def test_gradients_are_those_of_autograd(dtype, tol):
    """Against torch's automatic differentiation in 64 bits on the same numbers.  In fp32 some ten operators and products of sums of at
    most 96 terms follow each other, each off by (96 + 30) 2^-24 of the sums of its terms' sizes at most, which are up to three times the
    sums' own: 10 * 126 * 3 * 2^-24 = 2^-12.1 of a tensor's norm.  In bf16 activations and their gradients are rounded some nine times on
    the way, 2^-8 at most each, and the products add them up: 9 * 2^-8 * 2."""
    ex = _example()
    K, V, d, B, T = 2, 48, 32, 3, 40
    model, texts = ex.Model(K, V, d, 3, "cuda:0", dtype), ex.Texts(V, 2, 0.9, 3, "cuda:0")
    for name, f in (("g1", 1.3), ("g2", 0.7)):
        model.p[name].mul_(f)
    for name in ("b1", "b2"):
        model.p[name].add_(0.1)
    tok, target, first = texts.draw(K, B, T)
    loss = model.step(tok, target, first)
    for k in range(K):
        p = {n: (model.p[n][k] if n[0] in "gb" else model.copy[n][k]).double().cpu().requires_grad_() for n in model.p}
        want = _value(p, tok[k].cpu(), target[k].cpu(), first[k].cpu())
        want.backward()
        assert abs(float(loss[k]) - float(want.detach())) <= tol * float(want.detach())
        for name in p:
            got = model.grad[name][k].double().cpu()
            assert (got - p[name].grad).norm() <= tol * p[name].grad.norm(), name


def test_example_runs():
    """To its end; a text that is continued token by token has the states of the same text at once, up to the rounding of values and gates,
    2^-8 each, where products of one row and of several differ in it, of states of a size of four at most."""
    ex = _example()
    model, texts, losses, periods = ex.train(K=3, V=64, d=64, B=4, T=48, iterations=40)
    assert len(losses) == len(periods) and sum(periods) == 40 and all(l == l for l in losses)
    assert all(torch.equal(model.flat[0], model.flat[k]) for k in (1, 2))
    got = ex.continue_from(model, [5, 9], 6)
    text = [5, 9] + [t[0] for t in got]
    assert all(len(set(t)) == 1 for t in got) and len(text) == 8
    at_once, (_, _, _, s, _) = model.forward(torch.tensor(text[:-1], device="cuda").expand(3, 1, 7).contiguous())
    state = torch.zeros(3, 1, 64, device="cuda")
    for t in text[:-1]:
        _, (_, _, _, one, _) = model.forward(torch.full((3, 1, 1), t, device="cuda"), state=state, keep=False)
    assert one.last is state and torch.allclose(state, s.last, rtol=2.0 ** -6, atol=2.0 ** -6)


def test_step_recorded_and_replayed():
    """Forward and backward of a local step in a graph, replayed on other tokens between eager steps."""
    ex = _example()
    K, V, d, B, T = 2, 64, 32, 4, 40
    model, texts = ex.Model(K, V, d, 4, "cuda:0", torch.float32), ex.Texts(V, 2, 0.9, 4, "cuda:0")
    batch = texts.draw(K, B, T)
    model.step(*batch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model.step(*batch)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x = qsr_run(model, batch)
    for _ in range(3):
        for dst, src in zip(batch, texts.draw(K, B, T)):
            dst.copy_(src)
        want = [t.clone() for t in qsr_run(model, batch)]
        for t in x:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(x, want))


def qsr_run(model, batch):
    """The package's operators of a step, one behind the other, without the products between them."""
    import paper_2310_14423_amd as qsr
    tok, _, first = batch
    c, p = model.copy, model.p
    x = qsr.embedding(tok, c["E"])
    n = qsr.layernorm(x, p["g1"], p["b1"], residual=x)
    s = qsr.gated_scan(n.y, n.sum, reset=first, keep=True)
    dv, df, _ = qsr.gated_scan_backward(x, n.y, n.sum, s.states, reset=first)
    dx, dg, db = qsr.layernorm_backward(dv, n.sum, p["g1"], n.mean, n.rstd, residual_grad=df)
    return [x, n.y, n.sum, s.h, s.last, dv, df, dx, dg, db, qsr.embedding_backward(dx, tok, c["E"])]
