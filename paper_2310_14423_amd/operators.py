"""The operators around a caller's own matrix products (include/qsr.h): AdamW over many tensors, the root-mean-square norm with
the residual's addition, layer norm, the embedding, a gated linear recurrence, and the log probabilities of given tokens, each with its
gradients.

As in the binding, this is marshalling and the allocation of results and workspaces; nothing is computed in torch.  The calls that a
model makes in every step go through a small extension (csrc/torch_calls.cpp), the others through ctypes.  All of them work on the
current stream of the tensors' device, or on `stream` (a stream's address), which then also owns what they allocate.
Arguments that another stream owns have to be ready, and to be kept until the work is done, as for any of torch's own calls.
Shapes and types are checked here (ValueError), everything else in the library (QSRError).
None of them records a graph for automatic differentiation: the backward functions are called by hand, and where gradients are being
recorded a tensor that requires one is refused (ValueError) instead of being taken without it.
"""
import ctypes as C
from collections import namedtuple
from contextlib import ExitStack, nullcontext

from .binding import _check, lib

F32, BF16, E4M3 = 0, 1, 2       # QSR_TYPE_*
_nothing = nullcontext()
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


_torch = _calls = None


def _setup():
    """torch, and the extension that checks tensors, allocates and calls the library (csrc/torch_calls.cpp)."""
    global _torch, _calls
    import torch
    lib()               # fails loudly if nothing is built
    try:
        from . import _calls as calls
    except ImportError as e:
        raise RuntimeError("the operators' extension cannot be loaded: run `python -m paper_2310_14423_amd.build` (%s)" % e) from e
    calls.setup(_check, RMSNorm, TokenLogprobs, LayerNorm, GatedScan)
    _torch, _calls = torch, calls


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
        # (an ExternalStream at address 0 would be some other stream, and own what the default stream writes)
        side = torch.cuda.ExternalStream(stream, device=t.device) if stream else torch.cuda.default_stream(t.device)
        stack.enter_context(torch.cuda.stream(side))
    return (now if stream is None else stream), stack


def _need(ok, what):
    if not ok:
        raise ValueError(what)


# ---------------------------------------------------------------------------------------------------
# root-mean-square norm
# ---------------------------------------------------------------------------------------------------
RMSNorm = namedtuple("RMSNorm", "y sum rstd scale")


def rmsnorm(x, weight, residual=None, eps=1e-6, out="same", sum_out=None, stream=None):
    """y = s * rstd * weight for the rows of s = x + residual (or x); x [..., d] float32 or bfloat16, rows of any even stride;
    weight float32 [d], or [K][d] where x is [K][..., d], each worker's dense.  Returns (y, sum, rstd, scale):
      y      in x's type (out="same"), or float8_e4m3fn (out="fp8") with a float32 `scale` for each row (y = code * scale)
      sum    s in x's type, the residual stream behind (sum_out: a tensor for it, which may be x or residual); x itself
             where there is no residual
      rstd   1 / sqrt(mean(s^2) + eps), for the backward pass"""
    if _calls is None:
        _setup()
    _need(out == "same" or out == "fp8", "out: 'same' or 'fp8'")
    s, place = _place(x, stream)
    if place is None:
        return _calls.rmsnorm(x, weight, residual, eps, out == "fp8", sum_out, s)
    with place:
        return _calls.rmsnorm(x, weight, residual, eps, out == "fp8", sum_out, s)


def rmsnorm_backward(y_grad, sum, weight, rstd, residual_grad=None, stream=None):
    """(x_grad, weight_grad) of rmsnorm from its `sum` and `rstd`: x_grad, in the rows' type, is the gradient of x and of residual
    alike, with residual_grad (what comes down the residual stream) added; weight_grad is float32, shaped as weight."""
    if _calls is None:
        _setup()
    s, place = _place(sum, stream)
    if place is None:
        return _calls.rmsnorm_backward(y_grad, sum, weight, rstd, residual_grad, s)
    with place:
        return _calls.rmsnorm_backward(y_grad, sum, weight, rstd, residual_grad, s)


# ---------------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------------
LayerNorm = namedtuple("LayerNorm", "y sum mean rstd scale")


def layernorm(x, weight, bias=None, residual=None, eps=1e-5, out="same", sum_out=None, stream=None):
    """y = (s - mean(s)) * rstd * weight + bias for the rows of s = x + residual (or x), as rmsnorm takes and returns them: bias as weight,
    or None; the result (y, sum, mean, rstd, scale) with the rows' means and rstd = 1 / sqrt(mean((s - mean)^2) + eps), both float32."""
    if _calls is None:
        _setup()
    _need(out == "same" or out == "fp8", "out: 'same' or 'fp8'")
    s, place = _place(x, stream)
    if place is None:
        return _calls.layernorm(x, weight, bias, residual, eps, out == "fp8", sum_out, s)
    with place:
        return _calls.layernorm(x, weight, bias, residual, eps, out == "fp8", sum_out, s)


def layernorm_backward(y_grad, sum, weight, mean, rstd, residual_grad=None, bias=True, stream=None):
    """(x_grad, weight_grad, bias_grad) of layernorm from its `sum`, `mean` and `rstd`, as rmsnorm_backward has them; bias_grad is shaped
    as weight, or None with bias=False."""
    if _calls is None:
        _setup()
    s, place = _place(sum, stream)
    if place is None:
        return _calls.layernorm_backward(y_grad, sum, weight, mean, rstd, residual_grad, bool(bias), s)
    with place:
        return _calls.layernorm_backward(y_grad, sum, weight, mean, rstd, residual_grad, bool(bias), s)


# ---------------------------------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------------------------------
_TYPES = {"same": -1, "f32": F32, "bf16": BF16}


def embedding(tokens, table, scale=1.0, out="same", stream=None):
    """Rows scale * table[token] of a table [V][d], or [K][V][d] for tokens [K][...], each worker's its own: float32 or bfloat16, rows of
    any even stride.  tokens: int64, contiguous; outside 0..V-1: none, a row of zeros.  Returns tokens' shape + [d], in the table's type
    (out="same"), float32 ("f32") or bfloat16 ("bf16")."""
    if _calls is None:
        _setup()
    _need(out in _TYPES, "out: 'same', 'f32' or 'bf16'")
    s, place = _place(table, stream)
    if place is None:
        return _calls.embedding(tokens, table, scale, _TYPES[out], s)
    with place:
        return _calls.embedding(tokens, table, scale, _TYPES[out], s)


def embedding_backward(y_grad, tokens, table, scale=1.0, out=None, accumulate=False, stream=None):
    """The gradient of embedding's table for y_grad (float32 or bfloat16, rows of any even stride): scale times the sum of the rows of
    y_grad of each token, zero for the others, shaped and typed as table, of which nothing else is used.  out: a tensor for it, float32 or
    bfloat16, that shares no memory with y_grad and tokens (QSRError).  accumulate: it is added to what `out` holds (a table that the head
    shares, several batches); rows that no token names are left alone.  Sums are in a fixed order."""
    if _calls is None:
        _setup()
    s, place = _place(table, stream)
    if place is None:
        return _calls.embedding_backward(y_grad, tokens, table, scale, out, bool(accumulate), s)
    with place:
        return _calls.embedding_backward(y_grad, tokens, table, scale, out, bool(accumulate), s)


# ---------------------------------------------------------------------------------------------------
# gated linear recurrence
# ---------------------------------------------------------------------------------------------------
GatedScan = namedtuple("GatedScan", "h last states")
_INPUTS = {"complement": 0, "plain": 1}     # QSR_SCAN_*


def gated_scan(x, gate, initial=None, reset=None, lengths=None, input="complement", keep=False, state_out=None, stream=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t (input="complement") or a_t h_{t-1} + x_t ("plain") with a_t = sigmoid(gate_t), over the steps t of
    x and gate [..., T, d], for each channel by itself; float32 or bfloat16, each step's channels side by side, steps and sequences at any
    even stride (two parts of one product's output, time before batch).  States are float32.
      initial    [..., d]: h_{-1}; None: zeros
      reset      [..., T] bool: steps that take no state from before them (documents that are packed into one sequence)
      lengths    [...] int64: steps that there are; what is behind them is not read, h is 0 there
      keep       return `states` for the backward pass
      state_out  a float32 tensor [..., d] for `last`, which may be initial, and shares no memory with the arguments otherwise
    Returns (h, last, states): h in x's type, last [..., d] the states behind the sequences' ends, from which the next steps go on (one
    token at a time: T = 1), states or None."""
    if _calls is None:
        _setup()
    _need(input in _INPUTS, "input: 'complement' or 'plain'")
    s, place = _place(x, stream)
    if place is None:
        return _calls.gated_scan(x, gate, initial, reset, lengths, _INPUTS[input], bool(keep), state_out, s)
    with place:
        return _calls.gated_scan(x, gate, initial, reset, lengths, _INPUTS[input], bool(keep), state_out, s)


def gated_scan_backward(h_grad, x, gate, states, reset=None, lengths=None, last_grad=None, input="complement", stream=None):
    """(x_grad, gate_grad, initial_grad) of gated_scan for the gradients of h (in x's type) and of last (float32, or None: zero), from the
    same x, gate, reset, lengths and input and the `states` that were kept.  initial_grad is float32."""
    if _calls is None:
        _setup()
    _need(input in _INPUTS, "input: 'complement' or 'plain'")
    s, place = _place(x, stream)
    if place is None:
        return _calls.gated_scan_backward(h_grad, x, gate, states, reset, lengths, last_grad, _INPUTS[input], s)
    with place:
        return _calls.gated_scan_backward(h_grad, x, gate, states, reset, lengths, last_grad, _INPUTS[input], s)


# ---------------------------------------------------------------------------------------------------
# log probabilities of given tokens
# ---------------------------------------------------------------------------------------------------
TokenLogprobs = namedtuple("TokenLogprobs", "logp entropy lse stats top_logp top_id")


def token_logprobs(logits, tokens, top=0, temperature=1.0, stream=None):
    """For each row of logits [..., V] (float32 or bfloat16, rows of any even stride), z = logits / temperature: the log probability
    of its token (int64; outside 0..V-1: none, 0), the entropy, lse = log sum exp z, `stats` for the backward pass, and the `top`
    most probable tokens' log probabilities and ids (None with top = 0).  All results are float32, ids int32."""
    if _calls is None:
        _setup()
    s, place = _place(logits, stream)
    if place is None:
        return _calls.token_logprobs(logits, tokens, top, temperature, s)
    with place:
        return _calls.token_logprobs(logits, tokens, top, temperature, s)


def token_logprobs_backward(logits, tokens, stats, entropy, logp_grad=None, entropy_grad=None, temperature=1.0, out=None, stream=None):
    """The gradient with respect to logits, in their type, for float32 gradients of logp and of entropy (None: zero), from the
    forward pass's `stats` and `entropy` at the same temperature.  out: a tensor for it, which may be logits."""
    if _calls is None:
        _setup()
    s, place = _place(logits, stream)
    if place is None:
        return _calls.token_logprobs_backward(logits, tokens, stats, entropy, logp_grad, entropy_grad, temperature, out, s)
    with place:
        return _calls.token_logprobs_backward(logits, tokens, stats, entropy, logp_grad, entropy_grad, temperature, out, s)


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
    params: each of them once, also where a model uses one in two places.
    copies: bfloat16 tensors that get a copy of the new parameters, or None.
    weight_decay: one number, or one for each tensor.  clip_norm > 0: clipping by global norm over all tensors of a worker.
    moments: {"m": [...], "v": [...]} and with "fp8" also "m_scale", "v_scale" to go on with; zeros otherwise.  "f32": float32
    [K][n].  "fp8": float8_e4m3fn [K][whole blocks], scales float32 [K][blocks].  All of them are attributes m, v, m_scale, v_scale."""

    def __init__(self, params, grads, states="f32", copies=None, weight_decay=0.0, beta1=0.9, beta2=0.999, eps=1e-8, clip_norm=0.0,
                 seed=0, moments=None):
        self._handle = C.c_void_p()
        if _calls is None:
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
        # what a step writes: one tensor for each buffer, since views have their buffer's version
        wrote = params + (copies or []) + self.m + self.v + (self.m_scale or []) + (self.v_scale or [])
        self._written = tuple({id(t): t for t in (t._base if t._is_view() else t for t in wrote)}.values())
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
        cfg = AdamWConfig(K=self.K, n_tensors=len(params), grad_type=F32 if grads[0].dtype == torch.float32 else BF16,
                          state_type=E4M3 if states == "fp8" else F32, beta1=beta1, beta2=beta2, eps=eps, clip_norm=clip_norm,
                          seed=seed, tensors=arr)
        why = C.c_char_p()
        if lib().qsr_adamw_validate(C.byref(cfg), C.byref(why)) != 0:
            raise ValueError("AdamW: %s" % why.value.decode())
        _, place = _place(params[0], None)
        with place or _nothing:
            _check(lib().qsr_adamw_init(C.byref(cfg), C.byref(self._handle)), "qsr_adamw_init")

    def step(self, eta, t, stream=None):
        """One step of all workers with learning rate eta; t = steps taken before."""
        s, place = _place(self.params[0], stream)
        with place or _nothing:
            _calls.adamw_step(self._handle.value, t, eta, s, self._written)

    def set_grads(self, grads, stream=None):
        """Other tensors for the gradients, of the same type and strides, from the next step on."""
        grads = list(grads)
        _worker_rows(grads, self.params, (self.grads[0].dtype,), "grads")
        _need(all(g.shape[0] == 1 or g.stride(0) == h.stride(0) for g, h in zip(grads, self.grads)), "grads: strides stay")
        ptrs = (C.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
        s, place = _place(self.params[0], stream)
        with place or _nothing:
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
