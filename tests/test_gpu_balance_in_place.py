"""rr_balance_bwd with the gradient written over the scores, or added to them: bit for bit what separate buffers give."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E,k", [(1, 1), (5, 2), (8, 2), (64, 2), (100, 8), (256, 8)])
@pytest.mark.parametrize("S,L", [(1, 37), (7, 129), (4, 20000)])
def test_gradient_over_the_scores(E, k, S, L):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(E + S)
    a = 2 * torch.randn(S * L, E, generator=g, device="cuda")
    table = torch.topk(a, k, 1).indices.int().contiguous()
    live = torch.rand(S * L, generator=g, device="cuda") < 0.8
    _, count, n, _ = rr.balance_fwd(a, table, k, 0.4, 0.03, segments=S, live=live)
    want = rr.balance_bwd(a, count, n, k, 0.4, 0.03, live=live)
    over = a.clone()
    assert rr.balance_bwd(over, count, n, k, 0.4, 0.03, live=live, dlogits=over) is over and torch.equal(over, want)
    added = a.clone()
    rr.balance_bwd(added, count, n, k, 0.4, 0.03, live=live, dlogits=added, accumulate=True)
    assert torch.equal(added, torch.where(live[:, None], a + want, a))
