"""The example that runs the operators together: K workers train a next-token model with Local AdamW and QSR."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("local_adamw_tokens", os.path.join(ROOT, "examples", "local_adamw_tokens.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("states", ["f32", "fp8"])
def test_training_lowers_the_loss(states):
    """From log V, the loss of no knowledge (and a little more at the start), most of the way to the chain's entropy; the workers
    agree after the last round; the continuation follows the chain's likely successors."""
    ex = _example()
    V = 512
    model, chain, losses, periods = ex.train(K=3, V=V, T=300, states=states)
    entropy = -(0.9 + 0.1 / V) * math.log(0.9 + 0.1 / V) - (V - 1) * 0.1 / V * math.log(0.1 / V)
    assert len(losses) == len(periods) and sum(periods) == 300 and max(periods) > min(periods)
    assert losses[0] > 0.8 * math.log(V) and losses[-1] < entropy + 0.25 * (math.log(V) - entropy)
    assert all(torch.equal(model.flat[0], model.flat[k]) for k in (1, 2))
    tok = 5
    for nxt, alternatives in ex.continue_from(model, tok, 4):
        assert nxt == int(chain.next[tok]) and alternatives[0] > math.log(0.5) and alternatives == sorted(alternatives, reverse=True)
        tok = nxt


def test_gradients_are_those_of_autograd():
    """The example's backward pass against torch's automatic one in fp32 on the same bf16 numbers: activations and their gradients are
    rounded to bf16 some six times on the way, each 2^-8 at most, the products add them up: 5 % of a tensor's norm."""
    ex = _example()
    K, V, d, dh, n = 2, 64, 32, 64, 96
    model, chain = ex.Model(K, V, d, dh, 3, "cuda:0"), ex.Chain(V, 0.9, 3, "cuda:0")
    model.p["g1"].mul_(1.3)
    model.p["g2"].mul_(0.7)
    tok, target = chain.draw(K, n)
    loss = model.step(tok, target)
    for k in range(K):
        p = {name: (model.copy[name][k] if name not in ("g1", "g2") else model.p[name][k]).float().cpu().requires_grad_() for name in model.p}
        norm = lambda x, g: x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * g  # noqa: E731
        x = p["E"][tok[k].cpu()]
        z = norm(x + (norm(x, p["g1"]) @ p["W1"]).relu() @ p["W2"], p["g2"]) @ p["Wo"]
        want = torch.nn.functional.cross_entropy(z, target[k].cpu())
        want.backward()
        assert abs(float(loss[k]) - float(want.detach())) < 0.02 * float(want.detach())
        for name in p:
            got = model.grad[name][k].float().cpu()
            assert (got - p[name].grad).norm() <= 0.05 * p[name].grad.norm(), name
