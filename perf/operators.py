"""Timed cases of the operators around a caller's own matrix products: AdamW over many tensors, the root-mean-square norm
with the residual's addition, and the log probabilities of given tokens.

A language model that is trained with Local AdamW and QSR by its own backward pass has them in every local step, for K
workers at once; the norm in 8 bits and the log probabilities with alternatives are also what such a model is served with.

`run` computes a pass in elementary torch operations, in 32 bits, or (`own`) by the framework's entry points. Both work on
the same buffers:

  adamw   one flat buffer a kind, [K][total], in which the tensors of a worker start at multiples of 256 elements; the
          framework gets a view of each tensor. States in 8 bits are e4m3 codes with one scale for each 256 elements, and
          what is kept of the second moment is its square root.
  norm    rows [K][rows][d]
  tokens  logits [rows][V]
"""
import itertools
import math

import torch

own = False

DEV = "cuda:0"
BETA1, BETA2, EPS, DECAY, ETA = 0.9, 0.999, 1e-8, 0.05, 6e-4
BLOCK = 256                 # elements of a worker's tensor that share a scale
E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest step: one worker that trains the norms and biases of a 12-block encoder alone
        {"name": "adamw_vectors", "op": "adamw", "set": "vectors", "count": 72, "d": 768, "K": 1, "states": "f32",
         "grads": "f32", "clip": 0.0, "copies": False},
        # the perceptron's four tensors (784-1024-10), clipped, states in 8 bits
        {"name": "adamw_perceptron", "op": "adamw", "set": "perceptron", "d": 784, "d_hidden": 1024, "d_out": 10, "K": 8,
         "states": "fp8", "grads": "f32", "clip": 1.0, "copies": False},
        # ViT-B's encoder stack, 144 tensors, two workers, clipped, states in 32 bits
        {"name": "adamw_encoder_f32", "op": "adamw", "set": "encoder", "blocks": 12, "d": 768, "d_hidden": 3072, "K": 2,
         "states": "f32", "grads": "f32", "clip": 1.0, "copies": False},
        # the same stack on eight workers in mixed precision: gradients and the copies for the products in bf16, states in 8 bits
        {"name": "adamw_encoder_fp8", "op": "adamw", "set": "encoder", "blocks": 12, "d": 768, "d_hidden": 3072, "K": 8,
         "states": "fp8", "grads": "bf16", "clip": 0.0, "copies": True},
        # serving: the tokens of four sequences, one each, into an 8-bit product
        {"name": "norm_decode", "op": "norm", "K": 1, "rows": 4, "d": 2048, "type": "bf16", "out": "fp8", "train": False},
        # serving: a batch of prompts into an 8-bit product
        {"name": "norm_prompt", "op": "norm", "K": 1, "rows": 16384, "d": 4096, "type": "bf16", "out": "fp8", "train": False},
        # training: the encoder's tokens, 64 x 197 for each of eight workers, forward and backward
        {"name": "norm_train", "op": "norm", "K": 8, "rows": 12608, "d": 768, "type": "bf16", "out": "same", "train": True},
        # training in 32 bits, a width that is a multiple of nothing
        {"name": "norm_train_odd", "op": "norm", "K": 3, "rows": 1001, "d": 1003, "type": "f32", "out": "same", "train": True},
        # serving: one token of four sequences with eight alternatives
        {"name": "tokens_decode", "op": "tokens", "rows": 4, "V": 131072, "type": "bf16", "top": 8, "train": False},
        # scoring of texts in 32 bits, an odd vocabulary, five alternatives
        {"name": "tokens_score", "op": "tokens", "rows": 1001, "V": 50021, "type": "f32", "top": 5, "train": False},
        # training: loss and gradient of 16 sequences of 512 tokens
        {"name": "tokens_train", "op": "tokens", "rows": 8192, "V": 32768, "type": "bf16", "top": 0, "train": True},
        # training with few classes: eight workers' batches of 128 over 1000 classes in 32 bits
        {"name": "classes_train", "op": "tokens", "rows": 1024, "V": 1000, "type": "f32", "top": 0, "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adamw", "norm", "tokens"])
    while True:
        if op == "adamw":
            c = {"op": op, "set": rng.choice(["vectors", "perceptron", "encoder", "encoder"]), "K": rng.randint(1, 8),
                 "states": rng.choice(["f32", "fp8"]), "grads": rng.choice(["f32", "bf16"]), "clip": rng.choice([0.0, 1.0]),
                 "copies": rng.choice([False, True]), "d": _log(rng, 64, 1024)}
            if c["set"] == "vectors":
                c["count"] = _log(rng, 4, 300)
            elif c["set"] == "perceptron":
                c.update(d_hidden=_log(rng, 64, 2048), d_out=_log(rng, 2, 200))
            else:
                c.update(blocks=rng.randint(1, 12), d_hidden=_log(rng, c["d"], 4 * c["d"]))
        elif op == "norm":
            c = {"op": op, "K": rng.randint(1, 8), "rows": _log(rng, 1, 12608), "d": _log(rng, 64, 8192),
                 "type": rng.choice(["f32", "bf16"]), "out": "same", "train": rng.choice([False, True])}
            if not c["train"]:
                c["out"] = rng.choice(["same", "fp8"])
            if rng.random() < 0.5:
                c["d"] = max(64, c["d"] // 64 * 64)
        else:
            c = {"op": op, "rows": _log(rng, 1, 8192), "V": _log(rng, 500, 200000), "type": rng.choice(["f32", "bf16"]),
                 "top": 0, "train": rng.choice([False, True])}
            if not c["train"]:
                c["top"] = rng.choice([0, 1, rng.randint(2, 20)])
        if work(c)["bytes"] <= {"adamw": 1.09e10, "norm": 1.0e9, "tokens": 1.6e9}[op]:
            return c


# ---------------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------------
def _shapes(c):
    """The shapes of a worker's tensors."""
    d = c["d"]
    if c["set"] == "vectors":
        return [(d if i % 3 else 4 * d,) for i in range(c["count"])]
    if c["set"] == "perceptron":
        return [(d, c["d_hidden"]), (c["d_hidden"],), (c["d_hidden"], c["d_out"]), (c["d_out"],)]
    dh = c["d_hidden"]
    return [(d,), (d,), (d, 3 * d), (3 * d,), (d, d), (d,), (d,), (d,), (d, dh), (dh,), (dh, d), (d,)] * c["blocks"]


def work(case):
    c = case
    if c["op"] == "adamw":
        n = c["K"] * sum(math.prod(s) for s in _shapes(c))
        grad, state = (2 if c["grads"] == "bf16" else 4), (2 * (1 + 4 / BLOCK) if c["states"] == "fp8" else 8)
        return {"bytes": n * (8 + grad + 2 * state + (2 if c["copies"] else 0)), "flops": 16 * n}
    size = 2 if c["type"] == "bf16" else 4
    if c["op"] == "norm":
        n, rows, w = c["K"] * c["rows"] * c["d"], c["K"] * c["rows"], c["K"] * c["d"]
        b = 3 * size * n + (n + 4 * rows if c["out"] == "fp8" else size * n) + 4 * rows + 4 * w
        if c["train"]:      # the gradients of y and of the sum, the sum, and the gradient of both inputs; the weight and its gradient
            b += 4 * size * n + 4 * rows + 8 * w
        return {"bytes": b, "flops": n * (15 if c["train"] else 5)}
    n = c["rows"] * c["V"]
    b = size * n + c["rows"] * (8 + 12 + 8 * c["top"])
    if c["train"]:
        b += 2 * size * n + c["rows"] * (8 + 16)
    return {"bytes": b, "flops": n * (12 if c["train"] else 6)}


# ---------------------------------------------------------------------------------------------------
# preparation
# ---------------------------------------------------------------------------------------------------
def _codes(x):
    """e4m3 codes and scales of [K][blocks][256]."""
    scale = x.abs().amax(-1) * (1.0 / 448.0)
    q = (x / scale.clamp_min(1e-30)[..., None]).clamp_(-448.0, 448.0).to(E4M3)
    return q.view(x.shape[0], -1), scale


def _prepare_adamw(c, g):
    K, shapes = c["K"], _shapes(c)
    sizes = [math.prod(s) for s in shapes]
    blocks = [-(-n // BLOCK) for n in sizes]
    start = [BLOCK * b for b in itertools.accumulate([0] + blocks)]
    total = start.pop()
    at = torch.tensor(blocks, device=DEV)
    inside = torch.arange(total, device=DEV) - torch.tensor(start, device=DEV).repeat_interleave(at * BLOCK)
    inside = (inside < torch.tensor(sizes, device=DEV).repeat_interleave(at * BLOCK)).float()
    # matrices decay, vectors do not; every tensor has gradients of its own size
    decay = [DECAY if len(s) > 1 else 0.0 for s in shapes]
    sigma = (10.0 ** (-3.5 - 1.5 * torch.rand(len(shapes), generator=g, device=DEV))).repeat_interleave(at * BLOCK) * inside
    randn = lambda: torch.randn(K, total, generator=g, device=DEV)  # noqa: E731
    p = randn().mul_(0.02).mul_(inside)
    grad = randn().mul_(sigma).to(TYPES["bf16" if c["grads"] == "bf16" else "f32"])
    m = randn().mul_(0.3 * sigma)
    r = torch.rand(K, total, generator=g, device=DEV).add_(0.5).mul_(sigma)
    s = {"params": p, "grads": grad, "decay": torch.tensor(decay, device=DEV).repeat_interleave(at), "t": 1000, "seed": 17}
    if c["states"] == "fp8":
        s["m"], s["m_scale"] = _codes(m.view(K, -1, BLOCK))
        s["v"], s["v_scale"] = _codes(r.view(K, -1, BLOCK))
    else:
        s["m"], s["v"] = m, r.square_()
    if c["copies"]:
        s["copies"] = p.to(torch.bfloat16)
    if own:
        import paper_2310_14423_amd as qsr

        def views(flat, unit=1):
            return [flat[:, o // unit:o // unit + (n if unit == 1 else b)] for o, n, b in zip(start, sizes, blocks)]

        def padded(flat):
            return [flat[:, o:o + b * BLOCK] for o, b in zip(start, blocks)]

        if c["states"] == "fp8":
            moments = {"m": padded(s["m"]), "v": padded(s["v"]), "m_scale": views(s["m_scale"], BLOCK),
                       "v_scale": views(s["v_scale"], BLOCK)}
        else:
            moments = {"m": views(s["m"]), "v": views(s["v"])}
        s["opt"] = qsr.AdamW(views(p), views(grad), states=c["states"], copies=views(s["copies"]) if c["copies"] else None,
                             weight_decay=decay, beta1=BETA1, beta2=BETA2, eps=EPS, clip_norm=c["clip"], seed=s["seed"],
                             moments=moments)
    return s


def _prepare_norm(c, g):
    dt = TYPES[c["type"]]
    shape = (c["K"], c["rows"], c["d"])
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    # a residual stream whose rows differ in size, what a sub-block adds to it, and weights around one
    s = {"res": (randn(*shape) * torch.exp(randn(*shape[:2], 1))).to(dt), "x": randn(*shape).mul_(0.3).to(dt),
         "w": 1 + 0.1 * randn(c["K"], c["d"])}
    if c["train"]:
        s["dy"] = randn(*shape).mul_(1e-3).to(dt)
        s["dres"] = randn(*shape).mul_(1e-3).to(dt)
    return s


def _prepare_tokens(c, g):
    N, V, dt = c["rows"], c["V"], TYPES[c["type"]]
    x = torch.randn(N, V, generator=g, device=DEV).mul_(2.0)
    tok = torch.randint(0, V, (N,), generator=g, device=DEV)
    x.scatter_add_(1, tok[:, None], torch.full((N, 1), 6.0, device=DEV))
    if not c["train"]:          # tokens other than the given one that the grammar or a filter rules out, by either kind of mask
        given = x.gather(1, tok[:, None])
        cut = torch.randint(0, V, (N, max(1, V // 50)), generator=g, device=DEV)
        x.scatter_(1, cut, float("-inf"))
        x.scatter_(1, cut[:, ::2], torch.finfo(dt).min)
        x.scatter_(1, tok[:, None], given)
        if N >= 16:             # a row that is masked as a whole
            x[N // 3] = float("-inf")
    elif N >= 16:               # padding
        tok[N // 2:N // 2 + N // 16] = -1
    s = {"logits": x.to(dt), "tokens": tok}
    if c["train"]:
        s["dlogp"] = torch.full((N,), -1.0 / N, device=DEV)
        s["dent"] = torch.full((N,), -0.01 / N, device=DEV)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = {"adamw": _prepare_adamw, "norm": _prepare_norm, "tokens": _prepare_tokens}[case["op"]](case, g)
    s["case"] = dict(case)
    return s


# ---------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _adamw_outputs(s):
    return {k: s[k] for k in ("params", "m", "v", "m_scale", "v_scale", "copies") if k in s}


def _own_adamw(s):
    s["opt"].step(ETA, s["t"])
    s["t"] += 1
    return _adamw_outputs(s)


def _own_norm(s):
    import paper_2310_14423_amd as qsr
    c = s["case"]
    f = qsr.rmsnorm(s["x"], s["w"], residual=s["res"], eps=1e-6, out=c["out"])
    if not c["train"]:
        return {"y": f.y, "sum": f.sum, "rstd": f.rstd, "scale": f.scale} if c["out"] == "fp8" else \
            {"y": f.y, "sum": f.sum, "rstd": f.rstd}
    dx, dw = qsr.rmsnorm_backward(s["dy"], f.sum, s["w"], f.rstd, residual_grad=s["dres"])
    return {"y": f.y, "sum": f.sum, "rstd": f.rstd, "dx": dx, "dw": dw}


def _own_tokens(s):
    import paper_2310_14423_amd as qsr
    c = s["case"]
    f = qsr.token_logprobs(s["logits"], s["tokens"], top=c["top"])
    got = {"logp": f.logp, "entropy": f.entropy, "lse": f.lse}
    if c["top"]:
        got.update(top_logp=f.top_logp, top_id=f.top_id)
    if c["train"]:
        got["dlogits"] = qsr.token_logprobs_backward(s["logits"], s["tokens"], f.stats, f.entropy, s["dlogp"], s["dent"])
    return got


def _word(seed, t):
    """The step's 32-bit key: the high half of a 64-bit mix of seed and step."""
    z = (seed + (t + 1) * 0x9E3779B97F4A7C15) & (2 ** 64 - 1)
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & (2 ** 64 - 1)
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & (2 ** 64 - 1)
    return (z ^ (z >> 31)) >> 32


def _dither(seed, t, K, total):
    """Two random fractions in [0, 1) of 16 bits for each element of each worker: from a 32-bit mix of its index."""
    x = torch.arange(total, device=DEV)[None] + (torch.arange(K, device=DEV) * 0x9E3779B9)[:, None]
    x = (x ^ _word(seed, t)) & 0xFFFFFFFF
    x ^= x >> 16
    x = (x * 0x21F0AAAD) & 0xFFFFFFFF
    x ^= x >> 15
    x = (x * 0x735A2D97) & 0xFFFFFFFF
    x ^= x >> 15
    return (x >> 16).float() * 2.0 ** -16, (x & 0xFFFF).float() * 2.0 ** -16


def _round8(x, u, positive):
    """e4m3 codes of [K][blocks][256] by stochastic rounding with the fractions u, and the scales."""
    top = x.abs().amax(-1, keepdim=True)
    y = x * torch.where(top >= 1e-35, 448.0 / top, torch.zeros_like(top))
    if positive:        # what is not zero does not become zero
        y = torch.where(y > 0, y.clamp_min(2.0 ** -9), y)
    a = y.abs().clamp_max(448.0)
    exponent = (torch.frexp(a)[1] - 1).clamp_min(-6)
    step = torch.ldexp(torch.ones_like(a), exponent - 3)
    q = torch.copysign(torch.floor(a / step + u.view_as(a)) * step, y)
    scale = torch.where(top >= 1e-35, top * (1.0 / 448.0), torch.zeros_like(top))
    return q.to(E4M3).view(x.shape[0], -1), scale[..., 0]


def _plain_adamw(s):
    c, p = s["case"], s["params"]
    K, t = c["K"], s["t"] + 1
    blocks = lambda x: x.view(K, -1, BLOCK)  # noqa: E731
    g = blocks(s["grads"].float())
    if c["clip"] > 0:
        norm = g.square().sum((1, 2), dtype=torch.float32).sqrt()
        g = g * (c["clip"] / (norm + 1e-6)).clamp_max(1.0)[:, None, None]
    if c["states"] == "fp8":
        m, r = (blocks(s[k].float()) * s[k + "_scale"][..., None] for k in ("m", "v"))
        v = r * r
    else:
        m, v = blocks(s["m"]), blocks(s["v"])
    m = m + (1 - BETA1) * (g - m)
    v = v + (1 - BETA2) * (g * g - v)
    r = v.sqrt()
    step = (ETA / (1 - BETA1 ** t)) * m / (r * (1 / math.sqrt(1 - BETA2 ** t)) + EPS)
    theta = blocks(p)
    theta.sub_((ETA * s["decay"])[None, :, None] * theta + step)
    if c["states"] == "fp8":
        u, w = _dither(s["seed"], s["t"], K, p.shape[1])
        q, scale = _round8(m, u, False)
        s["m"].copy_(q)
        s["m_scale"].copy_(scale)
        q, scale = _round8(r, w, True)
        s["v"].copy_(q)
        s["v_scale"].copy_(scale)
    else:
        blocks(s["m"]).copy_(m)
        blocks(s["v"]).copy_(v)
    if c["copies"]:
        s["copies"].copy_(p)
    s["t"] += 1
    return _adamw_outputs(s)


def _plain_norm(s):
    c, dt, w = s["case"], s["x"].dtype, s["w"][:, None]
    h = s["x"].float() + s["res"].float()
    rstd = 1 / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    y = h * rstd * w
    got = {"sum": h.to(dt), "rstd": rstd[..., 0]}
    if c["out"] == "fp8":
        scale = y.abs().amax(-1, keepdim=True) * (1.0 / 448.0)
        got.update(y=(y / scale).clamp(-448.0, 448.0).to(E4M3), scale=scale[..., 0])
    else:
        got["y"] = y.to(dt)
    if c["train"]:
        h, dy = got["sum"].float(), s["dy"].float()
        u = dy * w
        dx = rstd * (u - h * (rstd * rstd * (u * h).mean(-1, keepdim=True))) + s["dres"].float()
        got.update(dx=dx.to(dt), dw=(dy * h * rstd).sum(1))
    return got


def _plain_tokens(s):
    c, tok = s["case"], s["tokens"]
    x = s["logits"].float()
    top = x.amax(-1, keepdim=True)
    z = x - top.clamp_min(torch.finfo(torch.float32).min)
    e = z.exp()
    total = e.sum(-1, keepdim=True)
    empty = (total == 0)[:, 0]
    lse = (top + total.log())[:, 0]
    lse = torch.where(empty, torch.full_like(lse, float("-inf")), lse)
    p = e / torch.where(total == 0, torch.ones_like(total), total)
    lp = torch.where(p > 0, z - total.log(), torch.zeros_like(z))
    entropy = -(p * lp).sum(-1)
    has = (tok >= 0) & (tok < c["V"])
    at = tok.clamp(0, c["V"] - 1)[:, None]
    logp = torch.where(empty, lse, x.gather(1, at)[:, 0] - lse)
    got = {"logp": torch.where(has, logp, torch.zeros_like(logp)), "entropy": entropy, "lse": lse}
    if c["top"]:        # the largest of pairs (value, the lower index first), in one whole number
        bits = x.view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = key * 2 ** 20 + (2 ** 20 - 1 - torch.arange(c["V"], device=DEV))
        ids = (2 ** 20 - 1) - (torch.topk(key, c["top"]).values & (2 ** 20 - 1))
        lpt = x.gather(1, ids) - lse[:, None]
        got.update(top_id=ids.int(), top_logp=torch.where(empty[:, None], lse[:, None].expand_as(lpt), lpt))
    if c["train"]:
        a = torch.where(has, s["dlogp"], torch.zeros_like(s["dlogp"]))[:, None]
        d = p * (-a - s["dent"][:, None] * (lp + entropy[:, None]))
        got["dlogits"] = d.scatter_add_(1, at, a).to(s["logits"].dtype)
    return got


_plain = {"adamw": _plain_adamw, "norm": _plain_norm, "tokens": _plain_tokens}
_own = {"adamw": _own_adamw, "norm": _own_norm, "tokens": _own_tokens}


# ---------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"adamw": _exact_adamw, "norm": _exact_norm, "tokens": _exact_tokens}[case["op"]](case, s)


def _exact_round8(x, u):
    """The e4m3 value below or above |x|, the upper one where the part of the step that is left exceeds 1 - u."""
    grid = torch.tensor([k * 2.0 ** -9 for k in range(8)] + [(8 + k) * 2.0 ** (e - 10) for e in range(1, 16) for k in range(8)][:-1],
                        dtype=torch.float64, device=DEV)
    a = x.abs().clamp(max=448.0)
    low = (torch.bucketize(a, grid, right=True) - 1).clamp(0, len(grid) - 2)
    below, above = grid[low], grid[low + 1]
    return torch.where((a - below) / (above - below) + u >= 1, above, below) * x.sign()


def _exact_adamw(c, s):
    K, n = c["K"], s["t"] + 1
    # (the random words are inputs: the same for everybody)
    words = _dither(s["seed"], s["t"], K, s["params"].shape[1]) if c["states"] == "fp8" else None
    got = {k: [] for k in _adamw_outputs(s)}
    shape = (-1, BLOCK)
    for k in range(K):
        g = s["grads"][k].double().view(shape)
        if c["clip"] > 0:
            g = g * min(1.0, c["clip"] / (float(g.pow(2).sum()) ** 0.5 + 1e-6))
        m, v = s["m"][k].double().view(shape), s["v"][k].double().view(shape)
        if c["states"] == "fp8":
            m, v = m * s["m_scale"][k].double()[:, None], (v * s["v_scale"][k].double()[:, None]).pow(2)
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g.pow(2)
        p = s["params"][k].double().view(shape)
        p = p - ETA * s["decay"].double()[:, None] * p - ETA * (m / (1 - BETA1 ** n)) / ((v / (1 - BETA2 ** n)).sqrt() + EPS)
        got["params"].append(p.view(-1))
        if c["states"] == "fp8":
            for name, x, u in (("m", m, words[0][k].double().view(shape)), ("v", v.sqrt(), words[1][k].double().view(shape))):
                top = x.abs().max(-1, keepdim=True).values
                y = torch.where(top > 0, 448 * x / top, 0 * x)
                if name == "v":
                    y = torch.where((y > 0) & (y < 2.0 ** -9), 0 * y + 2.0 ** -9, y)
                got[name].append(_exact_round8(y, u).view(-1))
                got[name + "_scale"].append(top[:, 0] / 448)
        else:
            got["m"].append(m.view(-1))
            got["v"].append(v.view(-1))
        if c["copies"]:
            got["copies"].append(p.view(-1))
    return {k: torch.stack(v) for k, v in got.items()}


def _exact_norm(c, s):
    w = s["w"].double().unsqueeze(1)
    h = s["x"].double() + s["res"].double()
    rms = (h.pow(2).sum(-1, keepdim=True) / c["d"] + 1e-6).sqrt()
    y = w * h / rms
    got = {"sum": h, "rstd": 1 / rms.squeeze(-1), "y": y}
    if c["out"] == "fp8":
        got["scale"] = y.abs().max(-1).values / 448
        got["y"] = y / got["scale"].unsqueeze(-1)
    if c["train"]:      # at the sum as it is kept; the row's norm stays that of the sum itself
        n, dy = h.to(s["x"].dtype).double() / rms, s["dy"].double()
        along = (dy * w * n).sum(-1, keepdim=True) / c["d"]
        got["dx"] = (dy * w - n * along) / rms + s["dres"].double()
        got["dw"] = (dy * n).sum(-2)
    return got


def _exact_tokens(c, s):
    x, tok = s["logits"].double(), s["tokens"]
    lse = torch.logsumexp(x, -1)
    empty = torch.isneginf(lse)
    lp = torch.where(empty.unsqueeze(-1), torch.full_like(x, float("-inf")), x - lse.unsqueeze(-1))
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    H = -plp.sum(-1)
    has = (tok >= 0) & (tok < c["V"])
    at = torch.where(has, tok, torch.zeros_like(tok)).unsqueeze(-1)
    got = {"logp": torch.where(has, lp.gather(1, at).squeeze(-1), torch.zeros_like(lse)), "entropy": H, "lse": lse}
    if c["top"]:
        v, i = torch.sort(x, dim=-1, descending=True, stable=True)
        got.update(top_logp=lp.gather(1, i[:, :c["top"]]), top_id=i[:, :c["top"]].int())
    if c["train"]:
        a = torch.where(has, s["dlogp"].double(), torch.zeros_like(lse)).unsqueeze(-1)
        d = torch.zeros_like(x).scatter_(1, at, a) - a * p
        got["dlogits"] = d - s["dent"].double().unsqueeze(-1) * (plp + p * H.unsqueeze(-1))
    return got
