"""The give-up path of the linear layer's kernels: with the waits for accumulators limited to one nanosecond they run out while the
tensor cores still work.  The kernel latches RR_ERR_TIMEOUT, every warp and the peer CTAs of its cluster leave their loops, TMEM is
given back and the kernel returns; nothing is broken and nothing hangs.  The next ordinary call on the same workspace is exact."""
import pytest
import torch

from graph_kernels import kernels

pytestmark = pytest.mark.gpu


def _ints(g, *shape):
    return torch.randint(-3, 4, shape, generator=g, device="cuda").bfloat16()


@pytest.fixture
def rr():
    import paper_2402_12399_b200 as rr
    yield rr
    rr.test_set_wait_limit_ns(0)


def _gives_up(rr, call, workspace):
    rr.test_set_wait_limit_ns(1)
    call()
    with pytest.raises(rr.RRError) as ei:
        rr.check(workspace)
    assert ei.value.code == 6
    rr.test_set_wait_limit_ns(0)
    rr.check(workspace)                     # the status has been handed over once


@pytest.mark.parametrize("M,N,K,kernel", [(5, 1024, 4096, "k_slim"), (100, 4096, 4096, "k_slim"), (600, 1024, 4096, "k_slim"),
                                          (300, 264, 8200, "k_slim"), (5000, 1032, 4096, "k_dense")])
def test_forward(rr, M, N, K, kernel):
    g = torch.Generator("cuda").manual_seed(M)
    x, w, b, r = _ints(g, M, K), _ints(g, N, K), _ints(g, N), _ints(g, M, N)
    y, z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    ws = rr.alloc_workspace(rr.linear_workspace_bytes(M, N, K)[0])

    def call():
        rr.linear_fwd(x, w, b, r, act=rr.ACT_RELU, out=y, z=z, workspace=ws)
    assert kernels(call) == [kernel]
    for _ in range(3):
        _gives_up(rr, call, ws)
        y.fill_(float("nan")), z.fill_(float("nan"))
        call()
        rr.check(ws)
        want = x.double() @ w.double().T + b.double()
        assert torch.equal(z, want.bfloat16()) and torch.equal(y, (want.clamp(min=0) + r.double()).bfloat16())


@pytest.mark.parametrize("M,N,K", [(64, 4096, 1024), (2048, 1032, 1024), (9000, 264, 520)])
def test_gradients(rr, M, N, K):
    g = torch.Generator("cuda").manual_seed(M)
    dy, x, w, z = _ints(g, M, N), _ints(g, M, K), _ints(g, N, K), _ints(g, M, N)
    dx, dw, db = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ws = rr.alloc_workspace(rr.linear_workspace_bytes(M, N, K)[1])

    def call():
        rr.linear_bwd(dy, x, w, z, act=rr.ACT_RELU, dx=dx, dw=dw, dbias=db, workspace=ws)
    assert "k_dense" in kernels(call) and ("k_slim" in kernels(call)) == (M <= 128)
    for _ in range(3):
        _gives_up(rr, call, ws)
        for t in (dx, dw, db):
            t.fill_(float("nan"))
        call()
        rr.check(ws)
        dz = dy.double() * (z > 0)
        assert torch.equal(dx, (dz @ w.double()).float()) and torch.equal(dw, (dz.T @ x.double()).float()) and torch.equal(db, dz.sum(0).float())
