"""Log probabilities of rows in which one token is nearly certain: what the many others come to is small beside it and must not be lost.

Tolerances.  U = 2^-24.  The sum s over e^((x - m)/T) is 1 for the largest logit and a small rest r.  The one trip of a lane that holds
the largest logit adds its terms in chains of at most four that are then joined in two steps: five roundings of a number near one, 5 U;
log s and the log probability take two more of their own size.  Everything else is a relative error of r: each factor 2^t on the way of a
term (its own and those by which a lane's, a wavefront's, a workgroup's and a part's sums come to a common m) has an exponent that is
off by 2 U of its size, 17 natural units together, and two units of its own: 2 * 17 + 2 * 6 = 46 U; sums of r's terms 10 U more.
So |log s - exact| <= 7 U + 60 U r, and 8 U + 64 U |logp| is allowed.  The entropy is log s plus (the mean of the distances), whose
terms carry their distances' roundings as well, in chains of sixteen: 8 U + 96 U H.  In the gradient the certain token's entry
a (1 - p) has the error of log s and the roundings of p and of the difference, 8 U + 4 U + 64 U |logp|, all times |a|."""
import numpy as np
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _exact(x, tok):
    z = x.double().cpu()
    rel = z - z.amax(-1, keepdim=True)
    e = rel.exp()
    rest = e.clone()
    rest.scatter_(1, rel.argmax(-1)[:, None], 0.0)
    ls = torch.log1p(rest.sum(-1))
    lp = rel - ls[:, None]
    return ls, lp.gather(1, tok.cpu()[:, None])[:, 0], -(lp.exp() * lp).sum(-1)


@pytest.mark.parametrize("above", [16.0, 16.5, 17.0])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top", [(2, 1000, 0), (600, 1000, 4), (3, 32768, 0), (600, 32768, 3), (2100, 32768, 0), (2, 131072, 0), (4, 131072, 8),
                                        (520, 131072, 0)])
def test_a_token_that_is_nearly_certain(rows, V, top, dt, above):
    """`above` over equal logits, each of whose terms is about half a unit of 1 in fp32 or less, wherever the certain token lies."""
    x = torch.zeros(rows, V, dtype=dt)
    tok = (torch.arange(rows) * 7919 + 5) % V
    x.scatter_(1, tok[:, None], above)
    x, tok = x.cuda(), tok.cuda()
    f = qsr.token_logprobs(x, tok, top=top)
    ls, logp, H = _exact(x[:8], tok[:8])
    p = logp.exp()
    got = f.stats.view(rows, 2)[:8, 1].double().cpu()
    assert (got - ls).abs().le(8 * U + 64 * U * ls).all(), float(((got - ls).abs() / U).max())
    assert (f.logp[:8].double().cpu() - logp).abs().le(8 * U + 64 * U * logp.abs()).all()
    assert (f.entropy[:8].double().cpu() - H).abs().le(8 * U + 96 * U * H).all()
    # all rows are alike but for the certain token's place
    assert (f.logp.double().cpu() - logp[0]).abs().le(8 * U + 64 * U * logp[0].abs()).all()
    a = torch.full((rows,), -1.0, device="cuda")
    d = qsr.token_logprobs_backward(x, tok, f.stats, f.entropy, a).gather(1, tok[:, None])[:8, 0].double().cpu()
    want, room = -(-torch.expm1(logp)), 12 * U + 64 * U * logp.abs()
    assert (d - want).abs().le(room + (2.0 ** -8 * want.abs() if dt == torch.bfloat16 else 0)).all()


@pytest.mark.parametrize("V", [1000, 32768, 131072])
def test_small_terms_of_many_sizes(V):
    """The certain token among logits of a normal distribution, at the row's start, in its middle and at its end, temperature 0.5."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn(6, V, generator=g) * 0.5 - 8.0
    tok = torch.tensor([0, V // 2, V - 1, 3, V // 3, V - 2])
    x.scatter_(1, tok[:, None], 0.25)
    f = qsr.token_logprobs(x.cuda(), tok.cuda(), temperature=0.5)
    ls, logp, H = _exact(x.double() * 2, tok)
    assert (f.logp.double().cpu() - logp).abs().le(8 * U + 64 * U * logp.abs()).all()
    assert (f.entropy.double().cpu() - H).abs().le(8 * U + 96 * U * H).all()
