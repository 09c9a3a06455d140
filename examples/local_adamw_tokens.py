"""Local AdamW with QSR on a small next-token model of the caller's own, for K workers on one GPU.

The model is an embedding, a residual sub-block and a head:

    x = E[token];  m = relu(norm(x) W1) W2;  logits = norm(x + m) Wo

Its matrix products are torch's, batched over the workers, on bf16 copies of the parameters.  Everything around them is this
package's: the embedding and its gradient, both norms with the residual's addition, log probabilities and their gradient, AdamW over all tensors at once (moments in
8 or in 32 bits, copies written by the same pass), the synchronization periods of Eq. (2) and the averaging of the workers.  Tokens
come from a random chain: each has one likely successor.

    python examples/local_adamw_tokens.py [--states fp8|f32] [--iterations N]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_14423_amd as qsr  # noqa: E402
from paper_2310_14423_amd.binding import make_config  # noqa: E402

BF16 = torch.bfloat16


class Chain:
    """Tokens whose successor is next[token] with probability `likely`, else any."""

    def __init__(self, V, likely, seed, dev):
        self.g = torch.Generator(device=dev)
        self.g.manual_seed(seed)
        self.V, self.likely, self.dev = V, likely, dev
        self.next = torch.randperm(V, generator=self.g, device=dev)

    def draw(self, *shape):
        r = lambda *s: torch.randint(0, self.V, s, generator=self.g, device=self.dev)  # noqa: E731
        tok, sure = r(*shape), torch.rand(*shape, generator=self.g, device=self.dev) < self.likely
        return tok, torch.where(sure, self.next[tok], r(*shape))


class Model:
    """K workers' parameters as views of one [K][P] buffer, their bf16 copies for the products, and gradients."""

    def __init__(self, K, V, d, dh, seed, dev):
        shapes = dict(E=(V, d), g1=(d,), W1=(d, dh), W2=(dh, d), g2=(d,), Wo=(d, V))
        sizes = [math.prod(s) for s in shapes.values()]
        P = sum(-(-n // 4) * 4 for n in sizes)
        self.flat = torch.zeros(K, P, device=dev)
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        self.p, self.copy, self.grad, at = {}, {}, {}, 0
        for (name, shape), n in zip(shapes.items(), sizes):
            view = self.flat[:, at:at + n].view(K, *shape)
            init = torch.ones(shape, device=dev) if len(shape) == 1 else torch.randn(shape, generator=gen, device=dev)
            view.copy_(init if name in ("E", "g1", "g2") else init / math.sqrt(shape[0]))      # the same for every worker
            self.p[name] = view
            self.copy[name] = view.to(BF16).contiguous()
            self.grad[name] = torch.zeros((K,) + shape, dtype=BF16, device=dev)
            at += -(-n // 4) * 4
        self.K, self.V, self.d = K, V, d

    def refresh(self):
        """The copies of parameters that something other than a step has changed."""
        for name, c in self.copy.items():
            c.copy_(self.p[name])

    def forward(self, tok):
        c = self.copy
        x = qsr.embedding(tok, c["E"])
        n1 = qsr.rmsnorm(x, self.p["g1"])
        a = torch.bmm(n1.y, c["W1"]).relu_()
        n2 = qsr.rmsnorm(torch.bmm(a, c["W2"]), self.p["g2"], residual=x)
        return x, n1, a, n2, torch.bmm(n2.y, c["Wo"])

    def step(self, tok, target):
        """Gradients of every worker's mean loss, and the losses."""
        turn = lambda t: t.transpose(1, 2).contiguous()  # noqa: E731
        c, g = self.copy, self.grad
        x, n1, a, n2, logits = self.forward(tok)
        lp = qsr.token_logprobs(logits, target)
        down = torch.full_like(lp.logp, -1.0 / tok.shape[1])
        dz = qsr.token_logprobs_backward(logits, target, lp.stats, lp.entropy, down, out=logits)
        torch.bmm(turn(n2.y), dz, out=g["Wo"])
        dm, dg2 = qsr.rmsnorm_backward(torch.bmm(dz, turn(c["Wo"])), n2.sum, self.p["g2"], n2.rstd)
        torch.bmm(turn(a), dm, out=g["W2"])
        da = torch.bmm(dm, turn(c["W2"])).mul_(a > 0)
        torch.bmm(turn(n1.y), da, out=g["W1"])
        dx, dg1 = qsr.rmsnorm_backward(torch.bmm(da, turn(c["W1"])), x, self.p["g1"], n1.rstd, residual_grad=dm)
        g["g1"].copy_(dg1)
        g["g2"].copy_(dg2)
        qsr.embedding_backward(dx, tok, c["E"], out=g["E"])
        return -lp.logp.mean(1)


def train(K=4, V=512, d=128, dh=256, tokens=1024, T=300, eta_max=3e-3, H_base=4, alpha=0.006, states="fp8", clip_norm=1.0, seed=1,
          dev="cuda:0", log=None):
    """Runs T iterations of Local AdamW under QSR.  Returns the model, the chain, the mean loss of each round's last iteration, and
    the rounds' periods."""
    eta = [eta_max * 0.5 * (1 + math.cos(math.pi * t / T)) for t in range(T)]
    w = dict(model="external", K=K, P=1, T=T, opt="adamw", H_base=H_base, alpha=alpha)
    cfg, keep = make_config(w, eta_table=eta)
    ends, periods = qsr.host_schedule(cfg)
    chain, model = Chain(V, 0.9, seed, dev), Model(K, V, d, dh, seed, dev)
    names = list(model.p)
    opt = qsr.AdamW([model.p[n] for n in names], [model.grad[n] for n in names], states=states, copies=[model.copy[n] for n in names],
                    weight_decay=[0.01 if n.startswith("W") else 0.0 for n in names], clip_norm=clip_norm, seed=seed)
    losses, ends = [], set(int(t) for t in ends)
    for t in range(T):
        loss = model.step(*chain.draw(K, tokens))
        opt.step(eta[t], t)
        if t + 1 in ends:           # the round's last local step: the workers are averaged
            qsr.average_rows(model.flat)
            model.refresh()
            losses.append(float(loss.mean()))
            if log:
                log("iteration %4d  round %3d of %3d iterations  loss %.3f" % (t + 1, len(losses), periods[len(losses) - 1], losses[-1]))
    opt.close()
    return model, chain, losses, list(periods)


def continue_from(model, first, n, top=3):
    """Greedy continuation of one token by worker 0, a token at a time, with each step's best alternatives: the head's input and
    weight in 8 bits."""
    W = model.p["Wo"][0].t()
    scale = W.abs().amax(1) / 448.0
    W8 = (W / scale[:, None]).to(torch.float8_e4m3fn)
    got, tok = [], torch.tensor([first], device=W.device)
    for _ in range(n):
        x = qsr.embedding(tok, model.copy["E"][0])
        a = (qsr.rmsnorm(x, model.p["g1"][0]).y @ model.copy["W1"][0]).relu_()
        y = qsr.rmsnorm(a @ model.copy["W2"][0], model.p["g2"][0], residual=x, out="fp8")
        logits = (y.y.float() @ W8.float().t()) * y.scale[:, None] * scale
        lp = qsr.token_logprobs(logits, tok, top=top)
        tok = lp.top_id[:, 0].long()
        got.append((int(tok), [round(float(v), 2) for v in lp.top_logp[0]]))
    return got


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--states", choices=("f32", "fp8"), default="fp8")
    ap.add_argument("--iterations", type=int, default=300)
    a = ap.parse_args()
    model, chain, losses, periods = train(T=a.iterations, states=a.states, log=print)
    print("%d rounds in %d iterations" % (len(periods), a.iterations))
    for tok, alternatives in continue_from(model, 0, 5):
        print("next", tok, "log probabilities of the best", alternatives)


if __name__ == "__main__":
    main()
