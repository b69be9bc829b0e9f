"""The linear layer where a CTA pair takes several tiles with several k-blocks each: the accumulators, the ring's stages and parities, the
staging tiles and what is requested ahead (bias, residual) are carried from tile to tile.  More than 148 tiles on 74 pairs, ragged
in all three sizes.  Each test asserts which kernel its sizes take.  Bounds as in test_gpu_linear.py."""
import functools

import numpy as np
import pytest
import torch

import block_ref as ref
from graph_kernels import kernels

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8
BF = dict(dtype=torch.bfloat16, device="cuda")
# tiles of 256 x 256 and k-blocks of 64: 17 x 17 of 9, 36 x 9 of 21, 79 x 2 of 5 (one row tile of the last band, one column of eight)
MANY = [(4099, 4104, 520), (9001, 2056, 1288), (20011, 264, 264)]


@functools.lru_cache(maxsize=2)
def _keep(seed, offset, M, N, p):
    keep, factor = ref.keep_mask(seed, offset, 0, M * N, p)
    return torch.from_numpy(keep.astype(np.uint8)).cuda().view(M, N).bool(), factor


def _drop(v, seed, offset, p):
    keep, factor = _keep(seed, offset, *v.shape, p)
    return torch.where(keep, v * factor, torch.zeros_like(v))


def _rng(seed, offset=3):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def _ints(g, *shape, most=3):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").bfloat16()


def _view(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _adder(n, magnitudes):
    return (n / 16 + 8) * 2.0 ** -23 * magnitudes


def _assert_within(got, want, tol, what=""):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


@pytest.mark.parametrize("M,N,K", MANY)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_whole_numbers_are_exact(M, N, K, dtype):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M + N)
    x, w, b, r = _ints(g, M, K), _ints(g, N, K), _ints(g, N, most=9), _ints(g, M, N, most=9).to(dtype)
    rng, z, y = _rng(M), torch.empty(M, N, **BF), torch.empty(M, N, dtype=dtype, device="cuda")
    ws = rr.alloc_workspace(rr.linear_workspace_bytes(M, N, K)[0])

    def call():
        rr.linear_fwd(x, w, b, r, act=rr.ACT_RELU, p=0.5, rng=rng, out=y, z=z, workspace=ws)
    assert kernels(call) == ["k_dense"]
    y.fill_(float("nan")), z.fill_(float("nan"))
    call()
    rr.check(ws)
    pre = x.double() @ w.double().T + b.double()
    assert torch.equal(z, pre.bfloat16())
    want = (r.double() + _drop(pre.clamp(min=0), M, 3, 0.5)).to(dtype)
    assert torch.equal(y, want)
    assert torch.equal(rr.linear_fwd(x, w, out_dtype=dtype), (pre - b.double()).to(dtype))
    same = r.clone()                                                 # in place of the residual
    rr.linear_fwd(x, w, b, same, act=rr.ACT_RELU, p=0.5, rng=rng, out=same, workspace=ws)
    assert torch.equal(same, want)
    # rows at the end of several tiles hold NaN and infinities
    odd = [0, 255, 256, M // 2, M - 1]
    x[odd] = torch.tensor([float("nan"), float("inf")], device="cuda").bfloat16().repeat(K // 2)
    call()
    rest = torch.ones(M, dtype=torch.bool)
    rest[odd] = False
    assert torch.equal(y[rest], want[rest]) and torch.isnan(z[odd]).all()
    rr.linear_fwd(x, w, residual=r, act=rr.ACT_GELU, p=1.0, rng=rng, out=y, workspace=ws)     # everything dropped
    assert torch.equal(y, r)


@pytest.mark.parametrize("M,N,K", MANY)
@pytest.mark.parametrize("act", range(5))
def test_forward(M, N, K, act):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M * 7 + act)
    pad = (0, 8, 24)[(M + act) % 3]
    x = _view(torch.randn(M, K, generator=g, device="cuda").bfloat16(), pad)
    w = (torch.randn(N, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    b = torch.randn(N, generator=g, device="cuda").bfloat16()
    z64 = x.double() @ w.double().T + b.double()
    mag = x.double().abs() @ w.double().abs().T + b.double().abs()
    v = ref.act(z64, act)
    for dtype in (torch.bfloat16, torch.float32):
        r = _view(torch.randn(M, N, generator=g, device="cuda").to(dtype), pad)
        z = _view(torch.empty(M, N, **BF), pad)
        wide = torch.full((M, N + pad), 5.0, dtype=dtype, device="cuda")
        y = rr.linear_fwd(x, w, b, r, act=act, p=0.1, rng=_rng(N), out=wide[:, :N], z=z)
        rr.check(y._workspace)
        assert torch.all(wide[:, N:] == 5.0)
        _assert_within(z, z64, HALF * z64.abs() + 2 * _adder(K, mag), "z")
        keep = _drop(torch.ones_like(v), N, 3, 0.1)
        want = v * keep + r.double()
        tol = torch.finfo(dtype).eps / 2 * want.abs() + keep * (1.2 * _adder(K, mag) + 3e-6 * (1 + z64.abs())) * 1.01 + 2.0 ** -22 * want.abs()
        _assert_within(y, want, tol, "y")


@pytest.mark.parametrize("M,N,K", [(4099, 4104, 520), (2500, 4104, 4104), (9001, 2056, 1288)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_in_whole_numbers_are_exact(M, N, K, dtype):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M)
    dy, x, w, z = _ints(g, M, N), _ints(g, M, K), _ints(g, N, K), _ints(g, M, N)
    dx, dw, db = torch.empty(M, K, dtype=dtype, device="cuda"), torch.empty(N, K, dtype=dtype, device="cuda"), torch.empty(N, device="cuda")
    rng, ws = _rng(M), rr.alloc_workspace(rr.linear_workspace_bytes(M, N, K)[1])

    def call(**kw):
        rr.linear_bwd(dy, x, w, z, act=rr.ACT_RELU, p=0.5, rng=rng, dx=dx, dw=dw, dbias=db, workspace=ws, **kw)
    assert kernels(call)[:2] == ["k_dz", "k_dense"]
    call()
    rr.check(ws)
    dz = _drop(dy.double(), M, 3, 0.5) * (z.double() > 0)
    want = (dz @ w.double(), dz.T @ x.double(), dz.sum(0))
    assert torch.equal(dx, want[0].to(dtype)) and torch.equal(dw, want[1].to(dtype)) and torch.equal(db, want[2].float())
    if dtype == torch.float32:
        call(add_dx=True, add_dw=True)
        assert torch.equal(dx, 2 * want[0].float()) and torch.equal(dw, 2 * want[1].float()) and torch.equal(db, 2 * want[2].float())


def test_calls_that_follow_at_once_see_each_other():
    """Chains on sizes of many tiles, with and without a synchronisation between the calls, and replayed from a graph."""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(1)
    M, N = 10000, 1032
    w, b = (torch.randn(N, N, generator=g, device="cuda") * N ** -0.5).bfloat16(), torch.randn(N, generator=g, device="cuda").bfloat16()
    start, rng = torch.randn(M, N, generator=g, device="cuda").bfloat16(), _rng(3, 0)
    fb, bb = rr.linear_workspace_bytes(M, N, N)
    ws, wb = rr.alloc_workspace(fb), rr.alloc_workspace(bb)
    x, y, z = torch.empty(M, N, **BF), torch.empty(M, N, **BF), torch.empty(M, N, **BF)
    dw, db = torch.empty(N, N, device="cuda"), torch.empty(N, device="cuda")

    def chain(wait=False):
        x.copy_(start), dw.zero_(), db.zero_()
        for i in range(6):
            for call in (lambda: rr.linear_fwd(x, w, b, x, act=rr.ACT_SILU, p=0.1, rng=rng, out=y, z=z, workspace=ws),
                         lambda: rr.linear_fwd(y, w, b, x, act=rr.ACT_GELU, out=x, workspace=ws),
                         lambda: rr.linear_bwd(x, y, w, z, act=rr.ACT_SILU, p=0.1, rng=rng, dx=z2, dw=dw, dbias=db, add_dw=True, workspace=wb),
                         lambda: rr.dropout_fwd(z2, 0.2, rng, residual=x, out=x)):
                call()
                if wait:
                    torch.cuda.synchronize()
            x.clamp_(-4, 4)
    z2 = torch.empty(M, N, **BF)

    def outputs():
        torch.cuda.synchronize()
        rr.check(ws), rr.check(wb)
        return [t.clone() for t in (x, y, z, z2, dw, db)]
    chain(True)
    want = outputs()
    assert all(torch.isfinite(t.float()).all() for t in want)
    chain()
    assert all(torch.equal(p, q) for p, q in zip(want, outputs()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(2):
        graph.replay()
    assert all(torch.equal(p, q) for p, q in zip(want, outputs()))


@pytest.mark.parametrize("M,N,K,kernel", [
    (1, 8, 8, "k_slim"), (128, 4096, 4096, "k_slim"), (129, 4104, 8, "k_dense"), (700, 648, 392, "k_slim"), (300, 2048, 4104, "k_slim"),
    (1111, 1416, 968, "k_dense"), (300, 4104, 264, "k_dense"), (20011, 24, 8, "k_dense"), (262400, 64, 8, "k_dense")])
def test_which_kernel_a_size_takes(M, N, K, kernel):
    """The sizes of the other tests cover both kernels; a change of the rule has to look at this coverage again."""
    import paper_2402_12399_b200 as rr
    x, w, y = torch.zeros(M, K, **BF), torch.zeros(N, K, **BF), torch.empty(M, N, **BF)
    ws = rr.alloc_workspace(rr.linear_workspace_bytes(M, N, K)[0])
    assert kernels(lambda: rr.linear_fwd(x, w, out=y, workspace=ws)) == [kernel]
