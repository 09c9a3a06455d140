"""The operators around a caller's own matrix products (include/qsr.h): AdamW over many tensors, the root-mean-square norm with
the residual's addition, and the log probabilities of given tokens, each with its gradients.

As in the binding, this is marshalling and the allocation of results and workspaces; nothing is computed in torch.  All of them
work on the current stream of the tensors' device, or on `stream` (a stream's address), which then also owns what they allocate.
Shapes and types are checked here (ValueError), everything else in the library (QSRError).
"""
import ctypes as C
from collections import namedtuple
from contextlib import ExitStack

from .binding import _check, lib

TYPES = {"f32": 0, "bf16": 1, "e4m3": 2}
BLOCK = 256     # elements that share a scale where moments are held in 8 bits


class Tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_int64), ("param_stride", C.c_int64),
                ("grad_stride", C.c_int64), ("state_stride", C.c_int64), ("scale_stride", C.c_int64), ("copy_stride", C.c_int64),
                ("weight_decay", C.c_double)]


class AdamWConfig(C.Structure):
    _fields_ = [("K", C.c_int32), ("n_tensors", C.c_int32), ("grad_type", C.c_int32), ("state_type", C.c_int32),
                ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("clip_norm", C.c_double),
                ("seed", C.c_uint64), ("tensors", C.POINTER(Tensor))]


class RMSNormArgs(C.Structure):
    _fields_ = [("K", C.c_int32), ("type", C.c_int32), ("y_type", C.c_int32), ("rows", C.c_int64), ("d", C.c_int64),
                ("x", C.c_void_p), ("residual", C.c_void_p), ("weight", C.c_void_p), ("sum", C.c_void_p), ("y", C.c_void_p),
                ("scale", C.c_void_p), ("rstd", C.c_void_p), ("x_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("sum_stride", C.c_int64), ("y_stride", C.c_int64), ("eps", C.c_double)]


class RMSNormBackwardArgs(C.Structure):
    _fields_ = [("K", C.c_int32), ("type", C.c_int32), ("rows", C.c_int64), ("d", C.c_int64), ("y_grad", C.c_void_p),
                ("sum", C.c_void_p), ("weight", C.c_void_p), ("rstd", C.c_void_p), ("residual_grad", C.c_void_p),
                ("x_grad", C.c_void_p), ("weight_grad", C.c_void_p), ("y_grad_stride", C.c_int64), ("sum_stride", C.c_int64),
                ("residual_grad_stride", C.c_int64), ("x_grad_stride", C.c_int64)]


class TokenLogprobsArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("stride", C.c_int64), ("type", C.c_int32), ("top", C.c_int32),
                ("logits", C.c_void_p), ("tokens", C.c_void_p), ("temperature", C.c_double), ("logp", C.c_void_p),
                ("entropy", C.c_void_p), ("lse", C.c_void_p), ("stats", C.c_void_p), ("top_logp", C.c_void_p), ("top_id", C.c_void_p)]


class TokenLogprobsBackwardArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("stride", C.c_int64), ("grad_stride", C.c_int64), ("type", C.c_int32),
                ("reserved", C.c_int32), ("logits", C.c_void_p), ("tokens", C.c_void_p), ("temperature", C.c_double),
                ("stats", C.c_void_p), ("entropy", C.c_void_p), ("logp_grad", C.c_void_p), ("entropy_grad", C.c_void_p),
                ("grad", C.c_void_p)]


_torch = _types = _functions = None


def _setup():
    """torch, the types of rows, and the library's functions with their argument types: looked up once."""
    global _torch, _types, _functions
    import torch
    L = lib()
    P, S, I32, I64, N = C.POINTER, C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    for name, args in (("qsr_rmsnorm", [P(RMSNormArgs), S]),
                       ("qsr_rmsnorm_workspace_bytes", [I32, I64, I64, I32, P(N)]),
                       ("qsr_rmsnorm_backward", [P(RMSNormBackwardArgs), S, N, S]),
                       ("qsr_token_logprobs_workspace_bytes", [I64, I64, I32, I32, P(N)]),
                       ("qsr_token_logprobs", [P(TokenLogprobsArgs), S, N, S]),
                       ("qsr_token_logprobs_backward", [P(TokenLogprobsBackwardArgs), S]),
                       ("qsr_adamw_step", [S, I64, C.c_double, S])):
        getattr(L, name).argtypes = args
    _types = {torch.float32: 0, torch.bfloat16: 1}
    _functions = L
    _torch = torch


def _place(t, stream):
    """(stream, None) where the tensor's device and the stream to work on are current; (stream, context) with what makes them so."""
    torch = _torch
    index = t.get_device()
    if index < 0:
        raise ValueError("tensors on a GPU are wanted, got one on %s" % t.device)
    here = index == torch.cuda.current_device()
    now = torch._C._cuda_getCurrentRawStream(index)         # (an object for the stream costs a microsecond)
    if here and (stream is None or stream == now):
        return now, None
    stack = ExitStack()
    if not here:
        stack.enter_context(torch.cuda.device(index))
    if stream is not None and stream != now:
        stack.enter_context(torch.cuda.stream(torch.cuda.ExternalStream(stream, device=t.device)))
    return (now if stream is None else stream), stack


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _type(t, what):
    ty = _types.get(t.dtype)
    if ty is None:
        raise ValueError("%s: float32 or bfloat16, got %s" % (what, t.dtype))
    return ty


def _row_stride(t, what):
    """Elements from row to row of a tensor [..., d] whose rows are dense and evenly spaced."""
    if t.is_contiguous():
        return t.shape[-1]
    sh, st = t.shape, t.stride()
    _need(sh[-1] == 1 or st[-1] == 1, "%s: the elements of a row lie side by side" % what)
    stride = expect = None
    for n, s in zip(reversed(sh[:-1]), reversed(st[:-1])):
        if n == 1:
            continue
        if stride is None:
            stride = s
        else:
            _need(s == expect, "%s: rows with one stride" % what)
        expect = s * n
    return sh[-1] if stride is None else stride


def _like(t, x, what):
    """A row argument's address and stride; it goes with the rows x."""
    if t.dtype != x.dtype or t.shape != x.shape or t.get_device() != x.get_device():
        raise ValueError("%s: shape, type and device of the rows" % what)
    return t.data_ptr(), _row_stride(t, what)


def _numbers(t, shape, x, what):
    """The address of float32 numbers, one or more for each row of x."""
    if t.dtype != _torch.float32 or t.shape != shape or not t.is_contiguous() or t.get_device() != x.get_device():
        raise ValueError("%s: contiguous float32 %s on the rows' device" % (what, tuple(shape)))
    return t.data_ptr()


# ---------------------------------------------------------------------------------------------------
# root-mean-square norm
# ---------------------------------------------------------------------------------------------------
RMSNorm = namedtuple("RMSNorm", "y sum rstd scale")


def _weight_rows(x, weight):
    """Workers and rows of each."""
    shape, of = x.shape, weight.shape
    _need(len(shape) >= 1 and 1 <= len(of) <= 2 and of[-1] == shape[-1] and weight.dtype == _torch.float32 and weight.is_contiguous()
          and weight.get_device() == x.get_device(), "weight: contiguous float32 [d] or [K][d]")
    K = of[0] if len(of) == 2 else 1
    _need(len(of) == 1 or (len(shape) >= 2 and shape[0] == K), "weight [K][d] goes with rows [K][...][d]")
    _need(K >= 1 and shape[-1] >= 1, "at least one worker and one element")
    return K, x.numel() // (K * shape[-1])


def rmsnorm(x, weight, residual=None, eps=1e-6, out="same", sum_out=None, stream=None):
    """y = s * rstd * weight for the rows of s = x + residual (or x); x [..., d] float32 or bfloat16, rows of any even stride;
    weight float32 [d], or [K][d] where x is [K][..., d].  Returns (y, sum, rstd, scale):
      y      in x's type (out="same"), or float8_e4m3fn (out="fp8") with a float32 `scale` for each row (y = code * scale)
      sum    s in x's type, the residual stream behind (sum_out: a tensor for it, which may be x or residual); x itself
             where there is no residual
      rstd   1 / sqrt(mean(s^2) + eps), for the backward pass"""
    if _torch is None:
        _setup()
    torch = _torch
    s, place = _place(x, stream)
    if place is not None:
        with place:
            return rmsnorm(x, weight, residual, eps, out, sum_out)
    ty = _type(x, "x")
    K, rows = _weight_rows(x, weight)
    shape = x.shape
    d = shape[-1]
    fp8 = out == "fp8"
    _need(fp8 or out == "same", "out: 'same' or 'fp8'")
    total = res_at = sum_at = None
    res_stride = sum_stride = 0
    if residual is not None:
        res_at, res_stride = _like(residual, x, "residual")
        total = torch.empty_like(x, memory_format=torch.contiguous_format) if sum_out is None else sum_out
    elif sum_out is not None:
        total = sum_out
    if total is not None:
        sum_at, sum_stride = _like(total, x, "sum_out")
    y = torch.empty_like(x, dtype=torch.float8_e4m3fn if fp8 else None, memory_format=torch.contiguous_format)
    rstd = torch.empty(shape[:-1], dtype=torch.float32, device=x.device)
    scale = torch.empty_like(rstd) if fp8 else None
    a = RMSNormArgs(K, ty, 2 if fp8 else ty, rows, d, x.data_ptr(), res_at, weight.data_ptr(), sum_at, y.data_ptr(),
                    scale.data_ptr() if fp8 else None, rstd.data_ptr(), _row_stride(x, "x"), res_stride, sum_stride, d, eps)
    _check(_functions.qsr_rmsnorm(a, s), "qsr_rmsnorm")
    return RMSNorm(y, x if total is None else total, rstd, scale)


def rmsnorm_backward(y_grad, sum, weight, rstd, residual_grad=None, stream=None):
    """(x_grad, weight_grad) of rmsnorm from its `sum` and `rstd`: x_grad, in the rows' type, is the gradient of x and of residual
    alike, with residual_grad (what comes down the residual stream) added; weight_grad is float32, shaped as weight."""
    if _torch is None:
        _setup()
    torch = _torch
    s, place = _place(sum, stream)
    if place is not None:
        with place:
            return rmsnorm_backward(y_grad, sum, weight, rstd, residual_grad)
    ty = _type(sum, "sum")
    K, rows = _weight_rows(sum, weight)
    shape = sum.shape
    d = shape[-1]
    dy_at, dy_stride = _like(y_grad, sum, "y_grad")
    res_at, res_stride = (None, 0) if residual_grad is None else _like(residual_grad, sum, "residual_grad")
    rstd_at = _numbers(rstd, shape[:-1], sum, "rstd")
    n = C.c_size_t(0)
    _check(_functions.qsr_rmsnorm_workspace_bytes(K, rows, d, ty, n), "qsr_rmsnorm_workspace_bytes")
    ws = torch.empty(n.value, dtype=torch.uint8, device=sum.device) if n.value else None
    x_grad, weight_grad = torch.empty_like(sum, memory_format=torch.contiguous_format), torch.empty_like(weight)
    a = RMSNormBackwardArgs(K, ty, rows, d, dy_at, sum.data_ptr(), weight.data_ptr(), rstd_at, res_at, x_grad.data_ptr(),
                            weight_grad.data_ptr(), dy_stride, _row_stride(sum, "sum"), res_stride, d)
    _check(_functions.qsr_rmsnorm_backward(a, None if ws is None else ws.data_ptr(), n, s), "qsr_rmsnorm_backward")
    return x_grad, weight_grad


# ---------------------------------------------------------------------------------------------------
# log probabilities of given tokens
# ---------------------------------------------------------------------------------------------------
TokenLogprobs = namedtuple("TokenLogprobs", "logp entropy lse stats top_logp top_id")


def _logit_rows(logits, tokens):
    """(rows' shape, number of rows, V)"""
    shape = logits.shape
    _need(len(shape) >= 1 and shape[-1] >= 1, "logits: [..., V]")
    _need(tokens.dtype == _torch.int64 and tokens.shape == shape[:-1] and tokens.is_contiguous() and
          tokens.get_device() == logits.get_device(), "tokens: contiguous int64, one for each row of logits")
    return shape[:-1], logits.numel() // shape[-1], shape[-1]


def token_logprobs(logits, tokens, top=0, temperature=1.0, stream=None):
    """For each row of logits [..., V] (float32 or bfloat16, rows of any even stride), z = logits / temperature: the log probability
    of its token (int64; outside 0..V-1: none, 0), the entropy, lse = log sum exp z, `stats` for the backward pass, and the `top`
    most probable tokens' log probabilities and ids (None with top = 0).  All results are float32, ids int32."""
    if _torch is None:
        _setup()
    torch = _torch
    s, place = _place(logits, stream)
    if place is not None:
        with place:
            return token_logprobs(logits, tokens, top, temperature)
    ty = _type(logits, "logits")
    shape, rows, V = _logit_rows(logits, tokens)
    dev, f32 = logits.device, torch.float32
    n = C.c_size_t(0)
    _check(_functions.qsr_token_logprobs_workspace_bytes(rows, V, ty, top, n), "qsr_token_logprobs_workspace_bytes")
    logp, entropy, lse = torch.empty((3,) + shape, dtype=f32, device=dev).unbind(0)
    stats = torch.empty(shape + (2,), dtype=f32, device=dev)
    top_logp = torch.empty(shape + (top,), dtype=f32, device=dev) if top else None
    top_id = torch.empty(shape + (top,), dtype=torch.int32, device=dev) if top else None
    ws = torch.empty(n.value, dtype=torch.uint8, device=dev) if n.value else None
    a = TokenLogprobsArgs(rows, V, _row_stride(logits, "logits"), ty, top, logits.data_ptr(), tokens.data_ptr(), temperature,
                          logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), stats.data_ptr(), top_logp.data_ptr() if top else None,
                          top_id.data_ptr() if top else None)
    _check(_functions.qsr_token_logprobs(a, None if ws is None else ws.data_ptr(), n, s), "qsr_token_logprobs")
    return TokenLogprobs(logp, entropy, lse, stats, top_logp, top_id)


def token_logprobs_backward(logits, tokens, stats, entropy, logp_grad=None, entropy_grad=None, temperature=1.0, out=None, stream=None):
    """The gradient with respect to logits, in their type, for float32 gradients of logp and of entropy (None: zero), from the
    forward pass's `stats` and `entropy` at the same temperature.  out: a tensor for it, which may be logits."""
    if _torch is None:
        _setup()
    s, place = _place(logits, stream)
    if place is not None:
        with place:
            return token_logprobs_backward(logits, tokens, stats, entropy, logp_grad, entropy_grad, temperature, out)
    ty = _type(logits, "logits")
    shape, rows, V = _logit_rows(logits, tokens)
    grad = _torch.empty_like(logits, memory_format=_torch.contiguous_format) if out is None else out
    grad_at, grad_stride = _like(grad, logits, "out")
    a = TokenLogprobsBackwardArgs(rows, V, _row_stride(logits, "logits"), grad_stride, ty, 0, logits.data_ptr(), tokens.data_ptr(),
                                  temperature, _numbers(stats, shape + (2,), logits, "stats"),
                                  _numbers(entropy, shape, logits, "entropy"),
                                  None if logp_grad is None else _numbers(logp_grad, shape, logits, "logp_grad"),
                                  None if entropy_grad is None else _numbers(entropy_grad, shape, logits, "entropy_grad"), grad_at)
    _check(_functions.qsr_token_logprobs_backward(a, s), "qsr_token_logprobs_backward")
    return grad


# ---------------------------------------------------------------------------------------------------
# AdamW over many tensors
# ---------------------------------------------------------------------------------------------------
def _worker_rows(ts, like, dtypes, what):
    _need(len(ts) == len(like), "%s: one for each parameter" % what)
    for t, p in zip(ts, like):
        _need(t.shape == p.shape and t.device == p.device and t.dtype in dtypes and t.dtype == ts[0].dtype and
              t.shape[0] >= 1 and t[0].numel() >= 1 and t[0].is_contiguous(),
              "%s: [K][...] as the parameters, each worker's part dense, of one type out of %s" % (what, dtypes))


class AdamW:
    """AdamW over a list of tensors [K][...] of K workers, float32, updated in place by step().

    grads: the gradients' tensors, float32 or bfloat16, read by every step (set_grads: other ones from then on).
    states: "f32" or "fp8" (moments in 8 bits: e4m3 codes in blocks of 256 elements with a scale, of m and of the root of v).
    copies: bfloat16 tensors that get a copy of the new parameters, or None.
    weight_decay: one number, or one for each tensor.  clip_norm > 0: clipping by global norm over all tensors of a worker.
    moments: {"m": [...], "v": [...]} and with "fp8" also "m_scale", "v_scale" to go on with; zeros otherwise.  "f32": float32
    [K][n].  "fp8": float8_e4m3fn [K][whole blocks], scales float32 [K][blocks].  All of them are attributes m, v, m_scale, v_scale."""

    def __init__(self, params, grads, states="f32", copies=None, weight_decay=0.0, beta1=0.9, beta2=0.999, eps=1e-8, clip_norm=0.0,
                 seed=0, moments=None):
        self._handle = C.c_void_p()
        if _torch is None:
            _setup()
        torch = _torch
        params, grads = list(params), list(grads)
        _need(params, "at least one tensor")
        _need(states in ("f32", "fp8"), "states: 'f32' or 'fp8'")
        _need(all(p.dim() >= 1 and p.shape[0] == params[0].shape[0] and p.device == params[0].device for p in params),
              "params: [K][...] with one K, on one device")
        _worker_rows(params, params, (torch.float32,), "params")
        _worker_rows(grads, params, (torch.float32, torch.bfloat16), "grads")
        if copies is not None:
            copies = list(copies)
            _worker_rows(copies, params, (torch.bfloat16,), "copies")
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * len(params)
        _need(len(decay) == len(params), "weight_decay: one number, or one for each tensor")
        self.K, self.dev = params[0].shape[0], params[0].device
        self.n = [p[0].numel() for p in params]
        self.states = states
        blocks = [-(-n // BLOCK) for n in self.n]
        code = torch.float8_e4m3fn if states == "fp8" else torch.float32
        sizes = [b * BLOCK for b in blocks] if states == "fp8" else self.n
        kinds = {"m": (sizes, code), "v": (sizes, code)}
        if states == "fp8":
            kinds.update(m_scale=(blocks, torch.float32), v_scale=(blocks, torch.float32))
        self.m_scale = self.v_scale = None
        for name, (size, dt) in kinds.items():
            if moments is None:
                flat = torch.zeros(self.K, sum(-(-s // 4) * 4 for s in size), dtype=torch.uint8 if dt is code and states == "fp8" else dt,
                                   device=self.dev).view(dt)
                at, got = 0, []
                for s in size:
                    got.append(flat[:, at:at + s])
                    at += -(-s // 4) * 4
            else:
                got = list(moments[name])
                _need(len(got) == len(params) and all(tuple(t.shape) == (self.K, s) and t.dtype == dt and t.device == self.dev and
                                                      (s == 1 or t.stride(1) == 1) for t, s in zip(got, size)),
                      "moments[%r]: %s [K][size], rows dense" % (name, dt))
            setattr(self, name, got)
        self.params, self.grads, self.copies = params, grads, copies
        stride = lambda t: t.stride(0)  # noqa: E731
        pairs = [(self.m, self.v)] + ([(self.m_scale, self.v_scale)] if states == "fp8" else [])
        _need(all(a.stride(0) == b.stride(0) for m, v in pairs for a, b in zip(m, v)), "moments: m and v with the same strides")
        arr = (Tensor * len(params))()
        for i, p in enumerate(params):
            t = arr[i]
            t.param, t.grad, t.m, t.v = p.data_ptr(), grads[i].data_ptr(), self.m[i].data_ptr(), self.v[i].data_ptr()
            t.n, t.param_stride, t.grad_stride, t.state_stride = self.n[i], stride(p), stride(grads[i]), stride(self.m[i])
            t.weight_decay = decay[i]
            if states == "fp8":
                t.m_scale, t.v_scale, t.scale_stride = self.m_scale[i].data_ptr(), self.v_scale[i].data_ptr(), stride(self.m_scale[i])
            if copies is not None:
                t.copy, t.copy_stride = copies[i].data_ptr(), stride(copies[i])
        cfg = AdamWConfig(K=self.K, n_tensors=len(params), grad_type=_type(grads[0], "grads"),
                          state_type=TYPES["e4m3"] if states == "fp8" else 0, beta1=beta1, beta2=beta2, eps=eps, clip_norm=clip_norm,
                          seed=seed, tensors=arr)
        why = C.c_char_p()
        if lib().qsr_adamw_validate(C.byref(cfg), C.byref(why)) != 0:
            raise ValueError("AdamW: %s" % why.value.decode())
        _, place = _place(params[0], None)
        with place or ExitStack():
            _check(lib().qsr_adamw_init(C.byref(cfg), C.byref(self._handle)), "qsr_adamw_init")

    def step(self, eta, t, stream=None):
        """One step of all workers with learning rate eta; t = steps taken before."""
        s, place = _place(self.params[0], stream)
        if place is not None:
            with place:
                return self.step(eta, t)
        _check(_functions.qsr_adamw_step(self._handle, t, eta, s), "qsr_adamw_step")

    def set_grads(self, grads, stream=None):
        """Other tensors for the gradients, of the same type and strides, from the next step on."""
        grads = list(grads)
        _worker_rows(grads, self.params, (self.grads[0].dtype,), "grads")
        _need(all(g.shape[0] == 1 or g.stride(0) == h.stride(0) for g, h in zip(grads, self.grads)), "grads: strides stay")
        ptrs = (C.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
        s, place = _place(self.params[0], stream)
        with place or ExitStack():
            _check(lib().qsr_adamw_set_grads(self._handle, ptrs, C.c_int32(len(grads)), C.c_void_p(s)), "qsr_adamw_set_grads")
        self.grads = grads

    def moments(self, i):
        """(m, v) of tensor i as float32 [K][n]."""
        if self.states == "f32":
            return self.m[i].clone(), self.v[i].clone()
        m, r = ((q[i].float().view(self.K, -1, BLOCK) * s[i][..., None]).flatten(1)[:, :self.n[i]]
                for q, s in ((self.m, self.m_scale), (self.v, self.v_scale)))
        return m, r * r

    def close(self):
        if self._handle:
            lib().qsr_adamw_destroy(self._handle)
            self._handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
