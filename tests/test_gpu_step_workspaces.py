"""The gradients of the norm and the embedding in a workspace that was made for a larger call: the same bits as in one of their own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large,small", [((131072, 1024), (131071, 1024)), ((131072, 1024), (65535, 1024)), ((65536, 1100), (65535, 1024)), ((5000, 256), (128, 256)),
                                         ((129, 8), (128, 8)), ((70000, 40), (16384, 33))])
def test_embedding_gradient(large, small):
    import paper_2402_12399_b200 as rr
    V, (n, d) = 700, small
    nbytes = rr.embed_workspace_bytes(large[0], V, large[1])[1]
    own = rr.embed_workspace_bytes(n, V, d)[1]
    assert own <= nbytes
    g = torch.Generator("cuda").manual_seed(n)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    ids[n // 3:] = 5          # most of them one id: every chunk leaves a piece
    dy = torch.randint(-3, 4, (n, d), generator=g, device="cuda").bfloat16()
    whole = torch.full((nbytes + 256,), 0x5a, dtype=torch.uint8, device="cuda")
    whole[:256] = 0
    got = rr.embed_bwd(ids, dy, torch.empty(V, d, device="cuda"), workspace=whole[:nbytes])
    rr.check(whole)
    assert torch.equal(got, rr.embed_bwd(ids, dy, torch.empty(V, d, device="cuda")))
    assert torch.equal(got, torch.zeros(V, d, device="cuda").index_add_(0, ids, dy.float()))     # (sums of small integers)
    # nothing is written behind the size that was asked for
    whole.fill_(0x5a)
    whole[:256] = 0
    assert torch.equal(got, rr.embed_bwd(ids, dy, torch.empty(V, d, device="cuda"), workspace=whole[:own]))
    assert (whole[own:] == 0x5a).all()


@pytest.mark.parametrize("large,small", [((16384, 4104), (16384, 4096)), ((700, 4104), (700, 4096)), ((700, 8200), (300, 4096)), ((2000, 1024), (1999, 1023))])
def test_norm_gradients(large, small):
    import paper_2402_12399_b200 as rr
    M, N = small
    nbytes = rr.norm_workspace_bytes(*large)
    g = torch.Generator("cuda").manual_seed(N)
    dy, h = (torch.randn(M, N, generator=g, device="cuda").bfloat16() for _ in range(2))
    mean, rstd = h.float().mean(1), 1 / h.float().std(1)
    whole = torch.full((nbytes + 256,), 0x5a, dtype=torch.uint8, device="cuda")
    whole[:256] = 0

    def call(ws):
        return rr.norm_bwd(dy, h, None, mean, rstd, dx=torch.empty_like(h), dw=torch.empty(N, device="cuda"), dbias=torch.empty(N, device="cuda"), workspace=ws)
    got = call(whole[:nbytes])
    assert all(torch.equal(a, b) for a, b in zip(got, call(None)))
    assert (whole[nbytes:] == 0x5a).all()
    # sums of M terms of either sign in at most 300 + M / 148 steps, each 2^-24 of the magnitudes
    want, size = dy.double().sum(0), dy.double().abs().sum(0)
    assert ((got[2].double() - want).abs() <= (300 + M / 148) * 2.0 ** -24 * size).all()


def test_calls_without_a_workspace_of_their_own():
    """The binding's own workspace has a header of zeros whatever its memory held before; what it holds behind does not matter."""
    import paper_2402_12399_b200 as rr
    n, V, d = 3000, 50, 4096
    g = torch.Generator("cuda").manual_seed(1)
    ids, dy = torch.randint(0, V, (n,), generator=g, device="cuda"), torch.randint(-3, 4, (n, d), generator=g, device="cuda").bfloat16()
    want = torch.zeros(V, d, device="cuda").index_add_(0, ids, dy.float())
    out, dw, rstd = torch.empty(V, d, device="cuda"), torch.empty(d, device="cuda"), torch.ones(n, device="cuda")
    for nbytes in (rr.embed_workspace_bytes(n, V, d)[1], rr.norm_workspace_bytes(n, d)):
        assert nbytes > 8 << 20
    sums = None
    for fill in (0, 0xff, 0x5a):
        for nbytes in (rr.embed_workspace_bytes(n, V, d)[1], rr.norm_workspace_bytes(n, d)):
            torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")      # goes back to the allocator, which hands it out again
        rr.embed_bwd(ids, dy, out)
        rr.check(out._workspace)
        assert torch.equal(out, want)
        rr.norm_bwd(dy, dy, None, None, rstd, kind=rr.NORM_RMS, dw=dw)
        sums = dw.clone() if sums is None else sums
        assert torch.equal(dw, sums)
    # an id outside the table is reported once, by the workspace that saw it
    ids[0] = V
    rr.embed_bwd(ids, dy, out)
    with pytest.raises(rr.RRError):
        rr.check(out._workspace)
