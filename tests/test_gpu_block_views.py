"""Views of one buffer that share no byte are taken, and those that do are refused, by the operators around the expert layer.
Whole numbers: the results are equal to those from separate buffers."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = dict(dtype=torch.bfloat16, device="cuda")


def _ints(g, *shape):
    return torch.randint(-3, 4, shape, generator=g, device="cuda").bfloat16()


@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (37, 64, 128), (300, 264, 72), (4500, 136, 64)])
def test_columns_of_one_buffer(M, N, K):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M)
    x, w, r, dy = _ints(g, M, K), _ints(g, N, K), _ints(g, M, N), _ints(g, M, N)
    z = torch.empty(M, N, **BF)
    y = rr.linear_fwd(x, w, residual=r, act=rr.ACT_RELU, z=z)
    dx, dw = torch.empty(M, K, **BF), torch.empty(N, K, **BF)
    rr.linear_bwd(dy, x, w, z, act=rr.ACT_RELU, dx=dx, dw=dw)
    wide = torch.full((M, 2 * K + 4 * N), 7.0, **BF)
    at = [0, K, K + N, K + 2 * N, K + 3 * N, K + 4 * N, 2 * K + 4 * N]
    vx, vr, vy, vz, vdy, vdx = (wide[:, a:b] for a, b in zip(at, at[1:]))
    vx.copy_(x), vr.copy_(r), vdy.copy_(dy)
    rr.linear_fwd(vx, w, residual=vr, act=rr.ACT_RELU, out=vy, z=vz)
    got = torch.empty(N, K, **BF)
    rr.linear_bwd(vdy, vx, w, vz, act=rr.ACT_RELU, dx=vdx, dw=got)
    for a, b in ((vx, x), (vr, r), (vy, y), (vz, z), (vdy, dy), (vdx, dx), (got, dw)):
        assert torch.equal(a, b)
    rr.linear_fwd(vx, w, residual=vr, act=rr.ACT_RELU, out=vr)       # in place of the residual, between its neighbours
    assert torch.equal(vr, y) and torch.equal(vx, x) and torch.equal(vy, y)
    for call in (lambda: rr.linear_fwd(vx, w, out=wide[:, K - 8:K - 8 + N]), lambda: rr.linear_fwd(vx, w, out=vy, z=wide[:, K + N + 8:K + 2 * N + 8]),
                 lambda: rr.linear_bwd(vdy, vx, w, vz, act=rr.ACT_RELU, dx=wide[:, at[5] - 8:at[6] - 8])):
        with pytest.raises(rr.RRError):
            call()


def test_what_is_not_read_may_be_written_over():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(3)
    M, N, K = 40, 64, 64
    x, w, dy = _ints(g, M, K), _ints(g, N, K), _ints(g, M, N)
    dx, dw = torch.empty(M, K, **BF), torch.empty(N, K, **BF)
    rr.linear_bwd(dy, x, w, dx=dx, dw=dw)
    x2, w2 = x.clone(), w.clone()
    rr.linear_bwd(dy, x2, w, dx=x2)                                  # x is read for dW alone
    rr.linear_bwd(dy, x, w2, dw=w2)                                  # and W for dx
    assert torch.equal(x2, dx) and torch.equal(w2, dw)
    for call in (lambda: rr.linear_bwd(dy, x, w, dx=dy), lambda: rr.linear_bwd(dy, x, w, dw=w, dx=dx), lambda: rr.linear_bwd(dy, x, w, dw=x[:0].new_empty(0)),
                 lambda: rr.linear_fwd(x, w, out=x), lambda: rr.linear_fwd(x, w, z=x), lambda: rr.linear_fwd(x, w, residual=dy, z=dy)):
        with pytest.raises((rr.RRError, ValueError)):
            call()


def test_dropout_in_one_buffer():
    import paper_2402_12399_b200 as rr
    both = torch.randn(2, 1000, device="cuda")
    rng = torch.tensor([1, 2], device="cuda")
    want = rr.dropout_fwd(both[0].clone(), 0.5, rng)
    assert torch.equal(rr.dropout_fwd(both[0], 0.5, rng, out=both[1]), want)
    flat = both.view(-1)
    for call in (lambda: rr.dropout_fwd(flat[:1000], 0.5, rng, out=flat[4:1004]), lambda: rr.dropout_fwd(flat[1000:], 0.5, rng, residual=flat[:1000], out=flat[4:1004]),
                 lambda: rr.dropout_bwd(flat[8:1008], 0.5, rng, out=flat[:1000], accumulate=True)):
        with pytest.raises(rr.RRError):
            call()
