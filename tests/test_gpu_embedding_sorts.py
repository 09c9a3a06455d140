"""The embedding's gradient by each way of sorting: one or two passes by one workgroup or by many, several rounds of a workgroup, chunks of 8
and of 32 tokens, and which of the two lists holds the result.

Rows of y_grad are whole numbers of at most 8 and scale is a power of two: sums of up to 2^21 of them are exact in fp32, in any order, and
the results are compared for equality."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu


def _tokens(kind, K, N, V, g):
    if kind == "spread":
        tok = torch.randint(0, V, (K, N), generator=g)
    else:                   # a few rows that most places name, some that one names, and the last row
        u = torch.rand(K, N, generator=g, dtype=torch.float64)
        tok = (torch.exp(u * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))) - 1).long().clamp_(0, V - 1)
    tok[:, N // 3:N // 3 + N // 20] = -1
    tok[:, -1] = V - 1
    return tok


def _check(K, N, V, d, kind, dt, grad_type, accumulate):
    g = torch.Generator().manual_seed(N + V)
    tok = _tokens(kind, K, N, V, g)
    dy = torch.randint(-8, 9, (K, N, d), generator=g)
    old = torch.randint(-100, 101, (K, V, d), generator=g)
    want = old.clone() if accumulate else torch.zeros(K, V, d, dtype=torch.int64)
    for k in range(K):
        some = tok[k] >= 0
        want[k].index_add_(0, tok[k][some], 4 * dy[k][some])
    out = old.to(grad_type).cuda()
    got = qsr.embedding_backward(dy.to(dt).cuda(), tok.cuda(), out, scale=4.0, out=out, accumulate=accumulate)
    # (a bf16 result is the exact sum rounded once)
    assert got is out and torch.equal(got.cpu(), want.to(torch.float32).to(grad_type))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["spread", "frequent"])
@pytest.mark.parametrize("K,N,V,d", [
    (1, 20000, 3000, 24), (2, 20000, 3000, 24), (1, 40000, 50021, 36), (2, 40000, 50021, 36),       # many workgroups, two passes: the second list
    (1, 20000, 300000, 16),                                                                         # three
    (1, 9000, 300, 40), (3, 9001, 511, 17),                                                         # one pass
    (1, 5000, 20000, 24), (2, 16384, 70000, 16),                                                    # one workgroup, two passes
    (1, 300000, 700, 8), (1, 300001, 200, 8), (2, 270001, 2100, 8),                                 # several rounds of a workgroup
])
def test_whole_numbers(K, N, V, d, kind, accumulate):
    _check(K, N, V, d, kind, torch.float32, torch.float32, accumulate)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("grad_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["spread", "frequent"])
@pytest.mark.parametrize("K,N,V,d", [(8, 9000, 4000, 520), (3, 30000, 2000, 260), (1, 70001, 600, 132)])
def test_long_chunks_of_bf16_rows(K, N, V, d, kind, grad_type, accumulate):
    """Chunks of 32 tokens, with rows in bf16 and several workers."""
    _check(K, N, V, d, kind, torch.bfloat16, grad_type, accumulate)
