"""Arguments in one piece of memory: refused where they share elements and may not, and right where their rows lie between each other's."""
import pytest
import torch

import paper_2310_14423_amd as qsr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V,d", [(6, 9, 16), (3000, 4000, 20)])
def test_rows_between_the_rows_of_a_table(N, V, d):
    """Whole numbers: exact in any order."""
    g = torch.Generator().manual_seed(1)
    both = torch.randint(-9, 10, (V, 3 * d), generator=g).float().cuda()
    dy, out, tok = both[:N, d + 3:2 * d + 3], both[:, :d], torch.randint(-1, V, (N,), generator=g).cuda()
    want = qsr.embedding_backward(dy.clone(), tok, out.clone())
    rest = both[:, d:].clone()
    assert qsr.embedding_backward(dy, tok, out, out=out) is out
    assert torch.equal(out, want) and torch.equal(both[:, d:], rest)
    for shared in (both[:N, d - 1:2 * d - 1], both[:N, 2 * d + 1:].as_strided((N, d), (3 * d, 1), 2 * d + 1), both.view(-1)[:N * d].view(N, d)):
        before = both.clone()
        with pytest.raises(qsr.QSRError) as e:
            qsr.embedding_backward(shared, tok, out, out=out)
        assert e.value.code == -1 and torch.equal(both, before)


def test_workers_with_a_token_each():
    """Tables and rows of y_grad in each worker's row of one buffer."""
    K, V, d = 3, 5, 8
    g = torch.Generator().manual_seed(2)
    flat = torch.randint(-9, 10, (K, V * d + d + 1), generator=g).float().cuda()
    out, dy, tok = flat[:, :V * d].view(K, V, d), flat[:, V * d:V * d + d].view(K, 1, d), torch.tensor([[1], [4], [-1]], device="cuda")
    want = qsr.embedding_backward(dy.clone(), tok, out.clone())
    qsr.embedding_backward(dy, tok, out, out=out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("T", [1, 40, 5000])
def test_states_beside_the_initial_ones(T):
    """In one buffer: side by side, the same, and one sequence on (refused)."""
    g = torch.Generator().manual_seed(3)
    x, f, states = torch.randn(3, T, 33, generator=g).cuda(), torch.randn(3, T, 33, generator=g).cuda(), torch.randn(6, 33, generator=g).cuda()
    want = qsr.gated_scan(x, f, initial=states[:3].clone())
    before = states.clone()
    for out in (states[1:4], states[2:5]):
        with pytest.raises(qsr.QSRError) as e:
            qsr.gated_scan(x, f, initial=states[:3], state_out=out)
        assert e.value.code == -1 and torch.equal(states, before)
    for out in (states[3:], states[:3]):
        got = qsr.gated_scan(x, f, initial=states[:3], state_out=out)
        assert got.last is out and torch.equal(out, want.last) and torch.equal(got.h, want.h)
