"""Argument checks of the operators around a caller's own products: nothing is launched on bad arguments, so no GPU is needed."""
import ctypes as C

import pytest

import operators_abi as ops
import paper_2310_14423_amd as qsr

P = 1 << 20         # an address that nothing reads


def _adamw(K=2, n=1000, **over):
    t = ops.Tensor(param=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, copy=P, n=n, param_stride=n, grad_stride=n,
                   state_stride=-(-n // 256) * 256, scale_stride=-(-n // 256), copy_stride=n, weight_decay=0.1)
    cfg = dict(K=K, n_tensors=1, grad_type=0, state_type=0, beta1=0.9, beta2=0.999, eps=1e-8, clip_norm=0.0, seed=0)
    for k, v in over.items():
        if k in cfg:
            cfg[k] = v
        else:
            setattr(t, k, v)
    arr = (ops.Tensor * 1)(t)
    return ops.AdamWConfig(tensors=arr, **cfg), arr


@pytest.mark.parametrize("over,why", [
    (dict(), None), (dict(state_type=2), None), (dict(grad_type=1, grad=P + 2, copy=P + 2), None), (dict(copy=None, copy_stride=0), None),
    (dict(K=1, param_stride=0, grad_stride=0, state_stride=0, scale_stride=0, copy_stride=0, state_type=2), None),
    (dict(K=0), "K"), (dict(K=65536), "K"), (dict(n_tensors=0), "tensors"), (dict(grad_type=2), "grad_type"),
    (dict(state_type=1), "state_type"), (dict(beta1=1.0), "beta1/beta2"), (dict(beta2=-0.1), "beta1/beta2"),
    (dict(beta2=float("nan")), "beta1/beta2"), (dict(eps=0.0), "eps"), (dict(eps=1e-39), "eps"), (dict(clip_norm=float("inf")), "clip_norm"),
    (dict(clip_norm=1e-60), "clip_norm"), (dict(n=0), "n"), (dict(n=1 << 36), "n"), (dict(param=None), "param"),
    (dict(param=P + 2), "param"), (dict(grad=P + 2), "grad"), (dict(grad_type=1, grad=P + 1), "grad"), (dict(m=None), "m/v"),
    (dict(v=P + 1), "m/v"), (dict(state_type=2, m_scale=None), "m_scale"), (dict(copy=P + 1), "copy"),
    (dict(param_stride=999), "param_stride"), (dict(grad_stride=0), "grad_stride"), (dict(copy_stride=5), "copy_stride"),
    (dict(state_stride=999), "state_stride"), (dict(state_type=2, state_stride=1000), "state_stride"),
    (dict(state_type=2, state_stride=1025), "state_stride"), (dict(state_type=2, scale_stride=3), "scale_stride"),
    (dict(weight_decay=float("nan")), "weight_decay"),
])
def test_adamw_configurations(over, why):
    cfg, keep = _adamw(**over)
    got, L = C.c_char_p(), qsr.lib()
    rc = L.qsr_adamw_validate(C.byref(cfg), C.byref(got))
    assert (rc, got.value) == (0, b"ok") if why is None else rc == -1 and why in got.value.decode()
    if why is not None:
        out = C.c_void_p(1)
        assert L.qsr_adamw_init(C.byref(cfg), C.byref(out)) == -1 and not out.value


def test_adamw_null_arguments():
    L = qsr.lib()
    assert L.qsr_adamw_validate(None, None) == -1 and L.qsr_adamw_init(None, None) == -1
    assert L.qsr_adamw_step(None, C.c_int64(0), C.c_double(0.1), None) == -1
    assert L.qsr_adamw_set_grads(None, None, C.c_int32(1), None) == -1
    assert L.qsr_adamw_clip(None, None, None) == -1 and L.qsr_adamw_destroy(None) == -1


def _norm(**over):
    a = dict(K=2, type=0, y_type=0, rows=3, d=100, x=P, residual=P, weight=P, sum=P, y=P, scale=P, rstd=P, x_stride=100,
             residual_stride=100, sum_stride=100, y_stride=100, weight_stride=100, eps=1e-6)
    a.update(over)
    return ops.RMSNormArgs(**a)


@pytest.mark.parametrize("over,code", [
    (dict(K=0), -1), (dict(rows=-1), -1), (dict(d=0), -1), (dict(d=16385, x_stride=20000, residual_stride=20000, sum_stride=20000, weight_stride=20000,
                                                               y_stride=20000), -7),
    (dict(type=2), -1), (dict(y_type=1), -1), (dict(y_type=3), -1), (dict(y_type=2, scale=None), -1), (dict(x=None), -1),
    (dict(x=P + 2), -1), (dict(residual=P + 1), -1), (dict(weight=None), -1), (dict(sum=P + 2), -1), (dict(y=None), -1),
    (dict(y=P + 2), -1), (dict(rstd=P + 2), -1), (dict(x_stride=99), -1), (dict(residual_stride=99), -1), (dict(sum_stride=0), -1),
    (dict(y_stride=99), -1), (dict(weight_stride=99), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(rows=0, x=None, y=None), 0),
])
def test_rmsnorm_arguments(over, code):
    a = _norm(**over)
    assert qsr.lib().qsr_rmsnorm(C.byref(a), None) == code


@pytest.mark.parametrize("over,ws,code", [
    (dict(rows=300), 0, -4), (dict(rows=300), 16, -4), (dict(rows=300), None, -1), (dict(type=2), 1 << 30, -1), (dict(y_grad=None), 1 << 30, -1), (dict(sum=P + 2), 1 << 30, -1),
    (dict(weight=None), 1 << 30, -1), (dict(rstd=None), 1 << 30, -1), (dict(residual_grad=P + 1), 1 << 30, -1),
    (dict(x_grad=None), 1 << 30, -1), (dict(weight_grad=None), 1 << 30, -1), (dict(x_grad_stride=99), 1 << 30, -1),
    (dict(y_grad_stride=99), 1 << 30, -1), (dict(sum_stride=99), 1 << 30, -1), (dict(residual_grad_stride=99), 1 << 30, -1),
    (dict(d=16385), 1 << 30, -1), (dict(weight_stride=99), 1 << 30, -1),
])
def test_rmsnorm_backward_arguments(over, ws, code):
    a = dict(K=2, type=0, rows=3, d=100, y_grad=P, sum=P, weight=P, rstd=P, residual_grad=P, x_grad=P, weight_grad=P, y_grad_stride=100,
             sum_stride=100, residual_grad_stride=100, x_grad_stride=100, weight_stride=100)
    a.update(over)
    a = ops.RMSNormBackwardArgs(**a)
    rc = qsr.lib().qsr_rmsnorm_backward(C.byref(a), C.c_void_p(0 if ws is None else P), C.c_size_t(ws or 0), None)
    assert rc == code


def test_rmsnorm_workspace():
    L, n = qsr.lib(), C.c_size_t(7)
    call = lambda K, rows, d, ty: L.qsr_rmsnorm_workspace_bytes(C.c_int32(K), C.c_int64(rows), C.c_int64(d), C.c_int32(ty), C.byref(n))  # noqa: E731
    assert call(0, 1, 1, 0) == -1 and n.value == 0
    assert call(1, 1, 16385, 0) == -7 and call(1, 1, 10, 2) == -1 and call(1, 1, 0, 0) == -1
    assert call(3, 1000, 768, 1) == 0 and n.value % (3 * 768 * 4) == 0 and n.value > 0


def _tokens(**over):
    a = dict(rows=3, vocab=100, stride=100, type=0, top=4, logits=P, tokens=P, temperature=1.0, logp=P, entropy=P, lse=P, stats=P,
             top_logp=P, top_id=P)
    a.update(over)
    return ops.TokenLogprobsArgs(**a)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), -1), (dict(vocab=0), -1), (dict(vocab=1 << 31, stride=1 << 31), -1), (dict(stride=99), -1), (dict(type=2), -1),
    (dict(top=-1), -1), (dict(top=65), -7), (dict(top=5, vocab=4), -1), (dict(logits=None), -1), (dict(logits=P + 2), -1),
    (dict(tokens=None), -1), (dict(tokens=P + 4), -1), (dict(temperature=0.0), -1), (dict(temperature=float("nan")), -1),
    (dict(temperature=1e60), -1), (dict(logp=P + 1), -1), (dict(stats=P + 2), -1), (dict(top_id=None), -1), (dict(top_logp=P + 2), -1),
    (dict(vocab=200000, stride=200000), -1), (dict(rows=0, logits=None), 0),
])
def test_token_logprobs_arguments(over, code):
    a = _tokens(**over)
    assert qsr.lib().qsr_token_logprobs(C.byref(a), None, C.c_size_t(0), None) == code


def test_token_logprobs_workspace():
    """Rows that are shared by workgroups need memory for the parts; enough rows, or short ones, need none."""
    L, n = qsr.lib(), C.c_size_t(7)
    call = lambda rows, V, ty, top: L.qsr_token_logprobs_workspace_bytes(C.c_int64(rows), C.c_int64(V), C.c_int32(ty), C.c_int32(top),  # noqa: E731
                                                                         C.byref(n))
    assert call(1, 0, 0, 0) == -1 and n.value == 0
    assert call(2, 200000, 0, 8) == 0 and n.value > 0
    a = _tokens(rows=2, vocab=200000, stride=200000, top=8)
    assert L.qsr_token_logprobs(C.byref(a), C.c_void_p(P), C.c_size_t(n.value - 1), None) == -4
    assert call(2, 100, 0, 8) == 0 and n.value == 0
    assert call(4096, 200000, 0, 8) == 0 and n.value == 0
    assert call(0, 100, 0, 8) == 0 and n.value == 0


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), -1), (dict(vocab=0), -1), (dict(stride=99), -1), (dict(grad_stride=99), -1), (dict(type=2), -1),
    (dict(temperature=-1.0), -1), (dict(logits=None), -1), (dict(grad=P + 2), -1), (dict(stats=None), -1), (dict(tokens=None), -1),
    (dict(entropy=None), -1), (dict(logp_grad=P + 2), -1), (dict(rows=0, logits=None), 0),
])
def test_token_logprobs_backward_arguments(over, code):
    a = dict(rows=3, vocab=100, stride=100, grad_stride=100, type=0, logits=P, tokens=P, temperature=1.0, stats=P, entropy=P, logp_grad=P,
             entropy_grad=P, grad=P)
    a.update(over)
    a = ops.TokenLogprobsBackwardArgs(**a)
    assert qsr.lib().qsr_token_logprobs_backward(C.byref(a), None) == code


def test_tensors_on_the_host_are_refused():
    import torch
    x, w = torch.zeros(3, 8), torch.ones(8)
    with pytest.raises(ValueError):
        qsr.rmsnorm(x, w)
    with pytest.raises(ValueError):
        qsr.token_logprobs(x, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        qsr.AdamW([x], [x])
