"""The operators' calls without a GPU: the streams that the Python side works on, and lists that name a tensor twice."""
import contextlib
import ctypes as C
import types

import pytest

import paper_2310_14423_amd as qsr
import paper_2310_14423_amd.operators as ops


class _Tensor:
    device = "cuda:1"

    def __init__(self, index=1):
        self.index = index

    def get_device(self):
        return self.index


def _torch(log, device=1, current=77):
    @contextlib.contextmanager
    def entered(what):
        log.append(what)
        yield
    cuda = types.SimpleNamespace(current_device=lambda: device, device=lambda i: entered(("device", i)), stream=entered,
                                 ExternalStream=lambda address, device: ("external", address), default_stream=lambda device: ("default", device))
    return types.SimpleNamespace(cuda=cuda, _C=types.SimpleNamespace(_cuda_getCurrentRawStream=lambda i: current))


@pytest.mark.parametrize("stream,want", [(0, ("default", "cuda:1")), (55, ("external", 55)), (77, None), (None, None)])
@pytest.mark.parametrize("device", [1, 0])
def test_streams(stream, want, device, monkeypatch):
    """Address 0 is the device's default stream: torch makes another stream of an external one at 0, which would then own the results
    that a kernel on the default stream writes."""
    log = []
    monkeypatch.setattr(ops, "_torch", _torch(log, device))
    s, place = ops._place(_Tensor(), stream)
    assert s == (77 if stream is None else stream)
    with place or contextlib.nullcontext():
        pass
    assert [x for x in log if x[0] != "device"] == ([want] if want else []) and [x for x in log if x[0] == "device"] == ([("device", 1)] if device == 0 else [])
    assert (place is None) == (not log)


def _list(n, state_type, **same):
    """n tensors of 300 elements for two workers at addresses of their own, but for those that are said to be the first one's."""
    arr = (ops.Tensor * n)()
    for i in range(n):
        t = arr[i]
        for j, name in enumerate(("param", "grad", "m", "v", "m_scale", "v_scale", "copy")):
            setattr(t, name, ((j + 1) << 32) + 8192 * (0 if same.get(name) == i else i))
        t.n, t.param_stride, t.grad_stride, t.state_stride, t.scale_stride, t.copy_stride = 300, 300, 300, 512, 2, 300
    return ops.AdamWConfig(K=2, n_tensors=n, grad_type=0, state_type=state_type, beta1=0.9, beta2=0.999, eps=1e-8, clip_norm=0.0, seed=0,
                           tensors=arr), arr


@pytest.mark.parametrize("state_type", [0, 2])
@pytest.mark.parametrize("name,refused", [("param", True), ("m", True), ("v", True), ("copy", True), ("m_scale", None), ("v_scale", None), ("grad", False)])
def test_tensors_named_twice(name, refused, state_type):
    """What a step writes is refused (scales only where there are any); gradients are only read."""
    refused = state_type == 2 if refused is None else refused
    for n, again in ((2, 1), (5, 3), (300, 299)):
        cfg, keep = _list(n, state_type, **{name: again})
        why = C.c_char_p()
        rc = qsr.lib().qsr_adamw_validate(C.byref(cfg), C.byref(why))
        assert rc == (-1 if refused else 0) and (not refused or (name + " (given twice)") in why.value.decode())
        cfg, keep = _list(n, state_type)
        assert qsr.lib().qsr_adamw_validate(C.byref(cfg), None) == 0


@pytest.mark.parametrize("T,code", [(1e-30, 0), (4.3e-39, 0), (4.2e-39, -1), (3e-39, -1), (1e38, 0)])
def test_temperatures(T, code):
    """Exponents are to the base 2: log2(e) / T has to be a float, not only 1 / T, or the largest logit's 0 * inf is NaN.  (No rows:
    nothing is launched on what is accepted.)"""
    from operators_abi import TokenLogprobsArgs, TokenLogprobsBackwardArgs
    P = 1 << 20
    a = dict(rows=0, vocab=100, stride=100, type=0, logits=P, tokens=P, temperature=T, entropy=P, stats=P)
    f = TokenLogprobsArgs(top=0, logp=P, lse=P, **a)
    assert qsr.lib().qsr_token_logprobs(C.byref(f), None, C.c_size_t(0), None) == code
    b = TokenLogprobsBackwardArgs(grad=P, grad_stride=100, logp_grad=P, entropy_grad=P, **a)
    assert qsr.lib().qsr_token_logprobs_backward(C.byref(b), None) == code


@pytest.mark.parametrize("state_type", [0, 2])
def test_tensors_that_overlap(state_type):
    """Tensors side by side are taken, ones that share an element are not: for every kind at its own size of a row."""
    for name, row in (("param", 1200), ("m", 512 if state_type == 2 else 1200), ("v", 512 if state_type == 2 else 1200), ("copy", 600)) + \
            ((("m_scale", 8), ("v_scale", 8)) if state_type == 2 else ()):
        for off, want in ((row, 0), (row - (2 if name == "copy" else 4), -1), (4, -1)):
            cfg, arr = _list(3, state_type)
            setattr(arr[2], name, getattr(arr[0], name) + off)
            assert qsr.lib().qsr_adamw_validate(C.byref(cfg), None) == want, (name, off)
