"""Argument checks of layer norm, the embedding and the gated recurrence: nothing is launched on bad arguments, so no GPU is needed."""
import ctypes as C

import pytest

import layers_abi as abi
import paper_2310_14423_amd as qsr

P = 1 << 20         # an address that nothing reads
BIG = 1 << 40       # a workspace of any size


def _norm(**over):
    a = dict(K=2, type=0, y_type=0, rows=3, d=100, x=P, residual=P, weight=P, bias=P, sum=P, y=P, scale=P, mean=P, rstd=P, x_stride=100,
             residual_stride=100, sum_stride=100, y_stride=100, weight_stride=100, bias_stride=100, eps=1e-5)
    a.update(over)
    return abi.LayerNormArgs(**a)


@pytest.mark.parametrize("over,code", [
    (dict(K=0), -1), (dict(K=65536), -1), (dict(rows=-1), -1), (dict(d=0), -1), (dict(d=16385), -7), (dict(type=2), -1), (dict(y_type=1), -1),
    (dict(y_type=3), -1), (dict(y_type=2, scale=None), -1), (dict(x=None), -1), (dict(x=P + 2), -1), (dict(residual=P + 1), -1), (dict(weight=None), -1),
    (dict(weight=P + 1), -1), (dict(bias=P + 2), -1), (dict(sum=P + 2), -1), (dict(y=None), -1), (dict(y=P + 2), -1), (dict(mean=P + 1), -1),
    (dict(rstd=P + 2), -1), (dict(scale=P + 2), -1), (dict(x_stride=99), -1), (dict(residual_stride=99), -1), (dict(sum_stride=0), -1), (dict(y_stride=99), -1),
    (dict(weight_stride=99), -1), (dict(bias_stride=99), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(rows=0, x=None, y=None), 0),
])
def test_layernorm_arguments(over, code):
    a = _norm(**over)
    assert qsr.lib().qsr_layernorm(C.byref(a), None) == code


@pytest.mark.parametrize("over,ws,code", [
    (dict(rows=300), 0, -4), (dict(rows=300), 16, -4), (dict(rows=300), None, -1), (dict(type=2), BIG, -1), (dict(y_grad=None), BIG, -1),
    (dict(sum=P + 2), BIG, -1), (dict(weight=None), BIG, -1), (dict(mean=None), BIG, -1), (dict(rstd=P + 1), BIG, -1), (dict(residual_grad=P + 1), BIG, -1),
    (dict(x_grad=None), BIG, -1), (dict(weight_grad=None), BIG, -1), (dict(bias_grad=P + 2), BIG, -1), (dict(x_grad_stride=99), BIG, -1),
    (dict(y_grad_stride=99), BIG, -1), (dict(sum_stride=99), BIG, -1), (dict(residual_grad_stride=99), BIG, -1), (dict(weight_stride=99), BIG, -1),
    (dict(d=16385, x_grad_stride=20000, y_grad_stride=20000, sum_stride=20000, residual_grad_stride=20000, weight_stride=20000), BIG, -7),
])
def test_layernorm_backward_arguments(over, ws, code):
    a = dict(K=2, type=0, rows=3, d=100, y_grad=P, sum=P, weight=P, mean=P, rstd=P, residual_grad=P, x_grad=P, weight_grad=P, bias_grad=P,
             y_grad_stride=100, sum_stride=100, residual_grad_stride=100, x_grad_stride=100, weight_stride=100)
    a.update(over)
    a = abi.LayerNormBackwardArgs(**a)
    assert qsr.lib().qsr_layernorm_backward(C.byref(a), C.c_void_p(0 if ws is None else P), C.c_size_t(ws or 0), None) == code


def test_layernorm_workspace():
    L, n = qsr.lib(), C.c_size_t(7)
    call = lambda K, rows, d, ty: L.qsr_layernorm_workspace_bytes(C.c_int32(K), C.c_int64(rows), C.c_int64(d), C.c_int32(ty), C.byref(n))  # noqa: E731
    assert call(0, 1, 1, 0) == -1 and n.value == 0
    assert call(1, 1, 16385, 0) == -7 and call(1, 1, 10, 2) == -1 and call(1, 1, 0, 0) == -1
    assert call(3, 1000, 768, 1) == 0 and n.value % (3 * 2 * 768 * 4) == 0 and n.value > 0
    assert call(3, 1, 768, 1) == 0 and n.value == 0
    assert L.qsr_layernorm_workspace_bytes(1, 1, 1, 0, None) == -1
    assert L.qsr_layernorm(None, None) == -1 and L.qsr_layernorm_backward(None, None, C.c_size_t(0), None) == -1


@pytest.mark.parametrize("over,code", [
    (dict(K=0), -1), (dict(K=65536), -1), (dict(type=2), -1), (dict(y_type=2), -1), (dict(tokens_each=-1), -1), (dict(vocab=0), -1),
    (dict(vocab=1 << 31), -1), (dict(d=0), -1), (dict(d=(1 << 22) + 1), -1), (dict(tokens_each=(1 << 27) + 1), -7), (dict(scale=float("nan")), -1),
    (dict(scale=1e39), -1), (dict(table=None), -1), (dict(table=P + 2), -1), (dict(type=1, table=P + 1), -1), (dict(tokens=None), -1),
    (dict(tokens=P + 4), -1), (dict(y=None), -1), (dict(y=P + 2), -1), (dict(table_stride=9), -1), (dict(y_stride=9), -1),
    (dict(worker_stride=9), -1), (dict(tokens_each=0, table=None, tokens=None, y=None), 0),
])
def test_embedding_arguments(over, code):
    a = dict(K=2, type=0, y_type=0, tokens_each=3, vocab=7, d=10, table=P, tokens=P, y=P, table_stride=10, worker_stride=70, y_stride=10, scale=1.0)
    a.update(over)
    a = abi.EmbeddingArgs(**a)
    assert qsr.lib().qsr_embedding(C.byref(a), None) == code


@pytest.mark.parametrize("over,ws,code", [
    (dict(tokens_each=9000), None, -1), (dict(tokens_each=9000), 16, -4), (dict(K=0), BIG, -1), (dict(type=2), BIG, -1), (dict(grad_type=2), BIG, -1), (dict(accumulate=2), BIG, -1),
    (dict(tokens_each=-1), BIG, -1), (dict(tokens_each=(1 << 27) + 1), BIG, -7), (dict(vocab=0), BIG, -1), (dict(d=0), BIG, -1),
    (dict(scale=float("inf")), BIG, -1), (dict(y_grad=None), BIG, -1), (dict(y_grad=P + 2), BIG, -1), (dict(tokens=None), BIG, -1),
    (dict(tokens=P + 4), BIG, -1), (dict(grad=None), BIG, -1), (dict(grad=P + 1), BIG, -1), (dict(y_grad_stride=9), BIG, -1),
    (dict(grad_stride=9), BIG, -1), (dict(worker_stride=69), BIG, -1), (dict(worker_stride=0), BIG, -1),
])
def test_embedding_backward_arguments(over, ws, code):
    """Among them workers whose tables share rows."""
    a = dict(K=2, type=0, grad_type=0, accumulate=0, tokens_each=3, vocab=7, d=10, y_grad=P, tokens=P, grad=P, y_grad_stride=10, grad_stride=10,
             worker_stride=70, scale=1.0)
    a.update(over)
    a = abi.EmbeddingBackwardArgs(**a)
    assert qsr.lib().qsr_embedding_backward(C.byref(a), C.c_void_p(0 if ws is None else P), C.c_size_t(ws or 0), None) == code


def test_embedding_workspace():
    L, n = qsr.lib(), C.c_size_t(7)
    call = lambda K, N, V, d, ty: L.qsr_embedding_workspace_bytes(C.c_int32(K), C.c_int64(N), C.c_int64(V), C.c_int64(d), C.c_int32(ty), C.byref(n))  # noqa: E731
    assert call(0, 1, 1, 1, 0) == -1 and n.value == 0
    assert call(1, 1, 1, 1, 2) == -1 and call(1, (1 << 27) + 1, 9, 8, 0) == -7
    assert call(1, 0, 9, 8, 0) == 0 and n.value == 0
    got = []
    for N in (1, 100, 4096, 4097, 100000, 1 << 27):
        assert call(2, N, 50000, 64, 1) == 0
        got.append(n.value)
    # few tokens need none; others the list of tokens and places, and a second one where a workgroup does not sort them alone
    assert got == sorted(got) and got[0] == got[1] == 0 and got[2] >= 2 * 8 * 4096 and got[4] >= 2 * 2 * 8 * 100000
    assert L.qsr_embedding(None, None) == -1 and L.qsr_embedding_backward(None, None, C.c_size_t(0), None) == -1


def _scan(cls, **over):
    a = dict(type=0, input=0, batch=3, steps=20, d=10, x=P, gate=P, reset=P, lengths=P, states=P)
    rows = ["x", "gate"]
    if cls is abi.GatedScanArgs:
        a.update(initial=P, h=P, last=P)
        rows.append("h")
    else:
        a.update(h_grad=P, last_grad=P, x_grad=P, gate_grad=P, initial_grad=P)
        rows += ["h_grad", "x_grad", "gate_grad"]
    a.update({n + "_stride": 10 for n in rows})
    a.update({n + "_batch_stride": 200 for n in rows})
    a.update(over)
    return cls(**a)


def _call(a, ws=BIG):
    f = qsr.lib().qsr_gated_scan if isinstance(a, abi.GatedScanArgs) else qsr.lib().qsr_gated_scan_backward
    return f(C.byref(a), C.c_void_p(0 if ws is None else P), C.c_size_t(ws or 0), None)


BOTH = [(dict(type=2), -1), (dict(input=2), -1), (dict(input=-1), -1), (dict(batch=-1), -1), (dict(steps=-1), -1), (dict(d=0), -1),
        (dict(steps=(1 << 30) + 1), -7), (dict(d=(1 << 28) + 1), -7), (dict(batch=1 << 31), -7), (dict(x=None), -1), (dict(x=P + 2), -1),
        (dict(gate=None), -1), (dict(gate=P + 1), -1), (dict(type=1, gate=P + 1), -1), (dict(lengths=P + 4), -1), (dict(states=P + 2), -1),
        (dict(x_stride=9), -1), (dict(gate_stride=9), -1), (dict(x_stride=(1 << 24) + 1), -7), (dict(gate_stride=1 << 40), -7), (dict(x_batch_stride=9), -1), (dict(gate_batch_stride=9), -1),
        (dict(batch=0, x=None), 0)]


@pytest.mark.parametrize("over,code", BOTH + [
    (dict(h=None), -1), (dict(h=P + 2), -1), (dict(initial=P + 2), -1), (dict(last=P + 1), -1), (dict(h_stride=9), -1), (dict(h_batch_stride=199), -1),
    (dict(h_stride=29, h_batch_stride=10), -1), (dict(h_stride=(1 << 24) + 1), -7), (dict(steps=0, last=None, x=None, gate=None, h=None), 0),
])
def test_gated_scan_arguments(over, code):
    """Among them rows of h that share elements, steps before sequences and the other way round."""
    assert _call(_scan(abi.GatedScanArgs, **over)) == code


@pytest.mark.parametrize("over,code", BOTH + [
    (dict(h_grad=None), -1), (dict(states=None), -1), (dict(x_grad=None), -1), (dict(gate_grad=P + 2), -1), (dict(last_grad=P + 2), -1),
    (dict(initial_grad=P + 1), -1), (dict(h_grad_stride=9), -1), (dict(h_grad_batch_stride=9), -1), (dict(x_grad_batch_stride=199), -1),
    (dict(gate_grad_stride=29, gate_grad_batch_stride=10), -1), (dict(h_grad_stride=(1 << 24) + 1), -7), (dict(x_grad_stride=(1 << 24) + 1), -7), (dict(steps=0, initial_grad=None, x=None), 0),
])
def test_gated_scan_backward_arguments(over, code):
    assert _call(_scan(abi.GatedScanBackwardArgs, **over)) == code


def test_gated_scan_workspace():
    """Few channels and many steps are cut into parts, for whose maps there has to be memory."""
    L, n = qsr.lib(), C.c_size_t(7)
    call = lambda B, T, d, ty: L.qsr_gated_scan_workspace_bytes(C.c_int64(B), C.c_int64(T), C.c_int64(d), C.c_int32(ty), C.byref(n))  # noqa: E731
    assert call(1, 1, 0, 0) == -1 and n.value == 0
    assert call(1, 1, 1, 2) == -1 and call(1, (1 << 30) + 1, 1, 0) == -7
    for B, T, d, parts in ((1, 1, 64, False), (1, 16, 64, False), (1, 100, 64, False), (1, 5000, 64, True), (1000, 5000, 64, False), (0, 5000, 64, False)):
        assert call(B, T, d, 0) == 0 and (n.value > 0) == parts
    assert call(1, 5000, 64, 0) == 0
    need = n.value
    over = dict(batch=1, steps=5000, d=64, **{k: 64 for k in ("x_stride", "gate_stride", "x_batch_stride", "gate_batch_stride")})
    for cls, rows in ((abi.GatedScanArgs, ["h"]), (abi.GatedScanBackwardArgs, ["h_grad", "x_grad", "gate_grad"])):
        a = _scan(cls, **over, **{r + s: 64 for r in rows for s in ("_stride", "_batch_stride")})
        assert _call(a, need - 1) == -4 and _call(a, None) == -1
    assert L.qsr_gated_scan(None, None, C.c_size_t(0), None) == -1 and L.qsr_gated_scan_backward(None, None, C.c_size_t(0), None) == -1


def test_tensors_on_the_host_are_refused():
    import torch
    x, w, tok = torch.zeros(3, 8), torch.ones(8), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: qsr.layernorm(x, w), lambda: qsr.layernorm_backward(x, x, w, x[:, 0], x[:, 0]), lambda: qsr.embedding(tok, x),
                 lambda: qsr.embedding_backward(x, tok, x), lambda: qsr.gated_scan(x, x), lambda: qsr.gated_scan_backward(x, x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_names_of_options():
    import torch
    x, w, tok = torch.zeros(3, 8), torch.ones(8), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: qsr.layernorm(x, w, out="bf16"), lambda: qsr.embedding(tok, x, out="fp8"), lambda: qsr.gated_scan(x, x, input="sum"),
                 lambda: qsr.gated_scan_backward(x, x, x, x, input=None)):
        with pytest.raises(ValueError, match="'"):
            call()
