"""rr_balance_fwd / rr_balance_bwd against the 64-bit statement.

Tolerances: counts are integers.  A softmax value is good to about 8 half steps of fp32 (exp 2, its argument's rounding |a - m| < 32
worth 2^-24 * 32 of the value at most, sum and reciprocal), and P sums fewer than 2^13 positive terms one after the other on any path
(tokens of a lane, then warps, then blocks), each adding 2^-24 relative: P, loss[0] within (64 + passes) 2^-24 < 1.6e-5 for the sizes
below; lse_i has an absolute error of a few 2^-24 |m|, so loss[1] the same relative bound.  A gradient element is
g_ij (cb (f_j - dot) + cz lse): its absolute error is a few 1e-6 of g_ij (cb max f + cz |lse|), bounded by 2e-5 of that."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
TOL = 1.6e-5


def _inputs(S, L, E, k, seed, live=None):
    g = torch.Generator("cuda").manual_seed(seed)
    a = torch.randn(S * L, E, generator=g, device="cuda") * 2 + torch.randn(E, generator=g, device="cuda")
    top = torch.topk(a, k, 1).indices.int()
    table = torch.cat([top, torch.full_like(top[:, :1], -1)], 1).contiguous()   # as the routing table: a further column
    if live == "ends":
        end = torch.randint(0, L + 1, (S,), generator=g, device="cuda")
        end[S // 2] = 0                                                          # one segment has no token
        live = (torch.arange(L, device="cuda")[None] < end[:, None]).reshape(-1)
    elif live == "none":
        live = torch.zeros(S * L, dtype=torch.bool, device="cuda")
    return a, table, live


def _check(a, table, k, S, live, alpha=0.4, beta=0.03, scale=-1.5):
    import paper_2402_12399_b200 as rr
    loss, count, n, P = rr.balance_fwd(a, table, k, alpha, beta, segments=S, live=live)
    rr.check(loss._workspace)
    l0, c0, n0, P0, d0 = ref.balance(torch.nan_to_num(a, 0, 0, 0) if live is not None else a, table, k, alpha, beta, S, live)
    assert torch.equal(count.cpu(), c0) and torch.equal(n.cpu(), n0)
    assert torch.allclose(P.double().cpu(), P0, rtol=TOL, atol=1e-12)
    assert torch.allclose(loss.double().cpu(), l0, rtol=TOL, atol=1e-12), (loss, l0)
    d = rr.balance_bwd(a, count, n, k, alpha, beta, scale=scale, live=live)
    clean = torch.nan_to_num(a.double().cpu(), 0, 0, 0)
    g = torch.softmax(clean, 1)
    T, E = a.shape
    seg = torch.arange(T) // max(1, T // S)
    nn = n0.clamp(min=1)[seg].double()
    segs, tokens = max(1, int((n0 > 0).sum())), max(1, int(n0.sum()))
    size = alpha * E / (segs * nn) * (c0.double()[seg].amax(1) / (k * nn)) + 2 * beta / tokens * torch.logsumexp(clean, 1).abs()
    assert torch.all((d.double().cpu() - scale * d0).abs() <= 2e-5 * abs(scale) * g * size[:, None] + 1e-30)
    if live is not None:
        assert torch.all(d[live == 0] == 0)
    before = torch.randn_like(a)
    acc = before.clone()
    rr.balance_bwd(a, count, n, k, alpha, beta, scale=scale, live=live, dlogits=acc, accumulate=True)
    assert torch.equal(acc, before + d)
    return loss, count, n, P, d


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (3, 1), (4, 2), (5, 5), (8, 2), (16, 4), (24, 3), (33, 2), (64, 2), (100, 8), (128, 1), (200, 8), (256, 8)])
@pytest.mark.parametrize("S,L", [(1, 1), (1, 37), (3, 700), (7, 129)])
def test_small_shapes(E, k, S, L):
    for live in (None, "ends"):
        _check(*_inputs(S, L, E, k, 31 * E + S, live)[:2], k, S, _inputs(S, L, E, k, 31 * E + S, live)[2])


def test_batch_of_padded_sequences_with_garbage_behind_their_ends():
    a, table, live = _inputs(32, 2048, 64, 2, 5, "ends")
    dead = ~live
    a[dead] = float("nan")
    a[dead.nonzero()[::3, 0]] = float("inf")
    a[dead.nonzero()[1::3, 0]] = torch.finfo(torch.float32).min
    table[dead] = 12345                                        # choices of what is no token are not looked at
    loss, count, n, P, d = _check(a, table, 2, 32, live)
    assert torch.isfinite(loss).all() and torch.isfinite(d).all()
    rr_live = live.to(torch.uint8) * 255                       # any non-zero value marks a token
    again = _check(a, table, 2, 32, rr_live)
    assert all(torch.equal(x, y) for x, y in zip((loss, count, n, P, d), again))   # and the results repeat


def test_masked_experts_of_live_tokens():
    """Scores at the type's lowest value: of some experts (they get nothing), and of a whole row (a uniform one; its log-sum-exp is out
    of range, so the z-loss is off)."""
    import paper_2402_12399_b200 as rr
    low = torch.finfo(torch.float32).min
    for E in (5, 8, 64):
        a, table, _ = _inputs(2, 300, E, 2, E)
        a[::7, : E // 2] = low
        a[5, 1:] = float("-inf")
        table = torch.topk(a, 2, 1).indices.int().contiguous()
        _check(torch.nan_to_num(a, neginf=low), table, 2, 2, None)
        first = rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=2)
        a[5, 1:] = low
        assert all(torch.equal(x, y) for x, y in zip(first, rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=2)))
        a[77] = low
        loss, count, n, P = rr.balance_fwd(a, table, 2, 0.1, segments=2)
        b = a.clone()
        b[77] = 0                                               # a uniform row like any other
        want = rr.balance_fwd(b, table, 2, 0.1, segments=2)
        assert torch.equal(P, want[3]) and torch.equal(loss, want[0]) and float(loss[1]) == 0
        assert torch.equal(rr.balance_bwd(a, count, n, 2, 0.1), rr.balance_bwd(b, count, n, 2, 0.1))


def test_many_and_few_segments():
    for S, L in ((4096, 3), (1, 65536), (592, 5), (1000, 1)):
        _check(*_inputs(S, L, 8, 2, S)[:2], 2, S, None)


def test_no_live_token_at_all():
    a, table, live = _inputs(4, 50, 16, 2, 9, "none")
    loss, count, n, P, d = _check(a, table, 2, 4, live)
    assert not loss.any() and not count.any() and not n.any() and not P.any() and not d.any()


def test_one_segment_and_first_choices_agree_with_the_older_loss():
    import paper_2402_12399_b200 as rr
    a, table, _ = _inputs(1, 5000, 32, 1, 8)
    loss, f, P = rr.aux_loss_fwd(a, table, 0.01)
    new = rr.balance_fwd(a, table, 1, 0.01)
    # (a division by a tensor: one by a number is a product with its rounded reciprocal, one rounding more than the kernel's)
    assert torch.equal(new[1][0].float() / torch.full_like(f, 5000), f) and torch.allclose(new[3][0], P, rtol=TOL) and torch.allclose(new[0][0], loss[0], rtol=TOL)
    assert torch.allclose(rr.balance_bwd(a, new[1], new[2], 1, 0.01), rr.aux_loss_bwd(a, f, 0.01), rtol=1e-4, atol=1e-10)


def test_choice_outside_the_experts_is_reported():
    import paper_2402_12399_b200 as rr
    a, table, _ = _inputs(2, 64, 8, 2, 1)
    table[70, 1] = 8
    table[71, 0] = -1
    loss, count, n, P = rr.balance_fwd(a, table, 2, 0.1, segments=2)
    with pytest.raises(rr.RRError):
        rr.check(loss._workspace)
    rr.check(loss._workspace)
    assert int(count.sum()) == 2 * 128 - 2


def test_empty_batch_and_reused_workspace():
    import paper_2402_12399_b200 as rr
    a, table, _ = _inputs(3, 0, 8, 2, 1)
    loss, count, n, P = rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=3)
    assert not loss.any() and not count.any() and not n.any() and not P.any()
    assert rr.balance_bwd(a, count, n, 2, 0.1).shape == (0, 8)
    ws = rr.alloc_workspace(rr.balance_workspace_bytes(4096, 64, 1))
    for S, L, E in ((1, 4096, 64), (4, 100, 64), (1, 4096, 64), (2, 30, 8)):
        a, table, _ = _inputs(S, L, E, 2, L)
        first = rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=S)
        again = rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=S, workspace=ws)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def test_captured():
    import paper_2402_12399_b200 as rr
    a, table, live = _inputs(4, 1000, 64, 2, 2, "ends")
    ws = rr.alloc_workspace(rr.balance_workspace_bytes(4000, 64, 4))
    d = torch.empty_like(a)

    def step():
        out = rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=4, live=live, workspace=ws)
        rr.balance_bwd(a, out[1], out[2], 2, 0.1, 0.1, live=live, dlogits=d)
        return out
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (3, 4):
        b, t, m = _inputs(4, 1000, 64, 2, seed, "ends")
        a.copy_(b), table.copy_(t), live.copy_(m)
        graph.replay()
        got = [x.clone() for x in out] + [d.clone()]
        want = list(step()) + [d]
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_binding_refuses():
    import paper_2402_12399_b200 as rr
    a, table, _ = _inputs(2, 64, 8, 2, 1)
    _, count, n, _ = rr.balance_fwd(a, table, 2, 0.1, segments=2)
    for call, err in [(lambda: rr.balance_fwd(a, table, 4, 0.1), rr.RRError),            # k above the table's width
                      (lambda: rr.balance_fwd(a, table, 0, 0.1), rr.RRError), (lambda: rr.balance_fwd(a, table, 2, 0.1, segments=3), rr.RRError),
                      (lambda: rr.balance_fwd(a.bfloat16(), table, 2, 0.1), TypeError), (lambda: rr.balance_fwd(a, table.long(), 2, 0.1), TypeError),
                      (lambda: rr.balance_fwd(a, table, 2, 0.1, live=torch.ones(5, dtype=torch.uint8, device="cuda")), TypeError),
                      (lambda: rr.balance_fwd(a, table, 2, 0.1, workspace=rr.alloc_workspace(256)), rr.RRError),
                      (lambda: rr.balance_fwd(a, table.cpu(), 2, 0.1), ValueError), (lambda: rr.balance_bwd(a, count.float(), n, 2, 0.1), TypeError),
                      (lambda: rr.balance_bwd(a, count, n, 2, 0.1, accumulate=True), ValueError)]:
        with pytest.raises(err):
            call()
