"""Arguments that share memory where they may not: refused on the host (no GPU is needed, nothing is launched)."""
import ctypes as C

import pytest

import layers_abi as abi
import paper_2310_14423_amd as qsr

P = 1 << 20         # an address that nothing reads


@pytest.mark.parametrize("over", [
    dict(y_grad=P), dict(y_grad=P + 4 * 10), dict(y_grad=P + 4 * 69), dict(y_grad=P - 4 * 9),           # 6 rows from, in, at the end of and before the first table
    dict(y_grad=P + 4 * 139), dict(y_grad=P + 4 * 70 - 4 * 5 * 10 - 4),                                 # the second table's last number; its first
    dict(type=1, y_grad=P + 2 * 279), dict(grad_type=1, y_grad=P + 2 * 139),                            # rows of another type
    dict(tokens=P), dict(tokens=P + 8 * 69), dict(tokens=P - 8 * 5),
    dict(accumulate=1, y_grad=P + 40),
    dict(worker_stride=1000, y_grad=P + 4 * 1000),                                                      # tables apart: the second
    dict(K=1, grad_stride=25, y_grad=P + 4 * 9, y_grad_stride=25), dict(K=1, grad_stride=25, y_grad=P + 4 * 16, y_grad_stride=25),   # rows beside rows
    dict(K=1, grad_stride=25, y_grad=P + 4 * 10, y_grad_stride=24),                                     # beside the first one, within the second
    dict(tokens_each=3000, y_grad=P + 4 * 10),                                                          # by a sort, too
    dict(y_grad=P + 4 * 69, y_grad_stride=1 << 62),
])
def test_gradient_of_a_table(over):
    a = dict(K=2, type=0, grad_type=0, accumulate=0, tokens_each=3, vocab=7, d=10, y_grad=P << 4, tokens=P << 5, grad=P, y_grad_stride=10,
             grad_stride=10, worker_stride=70, scale=1.0)
    a.update(over)
    a = abi.EmbeddingBackwardArgs(**a)
    assert qsr.lib().qsr_embedding_backward(C.byref(a), C.c_void_p(P << 6), C.c_size_t(1 << 40), None) == -1


@pytest.mark.parametrize("last", [P + 4, P - 4, P + 4 * 10, P - 4 * 29, P + 4 * 29])
@pytest.mark.parametrize("steps", [1, 20, 5000])
def test_states_that_are_partly_the_initial_ones(last, steps):
    a = abi.GatedScanArgs(type=0, input=0, batch=3, steps=steps, d=10, x=P << 4, gate=P << 5, h=P << 6, initial=P, last=last, x_stride=30, gate_stride=30, h_stride=30,
                          x_batch_stride=10, gate_batch_stride=10, h_batch_stride=10)
    assert qsr.lib().qsr_gated_scan(C.byref(a), C.c_void_p(P << 7), C.c_size_t(1 << 40), None) == -1
