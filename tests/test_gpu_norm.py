"""rr_norm_fwd / rr_norm_bwd against 64-bit arithmetic.

u = 2^-24.  A row's sums have at most 32 terms in a thread, 5 steps in a warp and 32 between warps: relative errors below 70 u of the sum of
magnitudes.  So rstd is off by at most 40 u of itself, the centre of a row by 70 u of its spread; y by half a step of its type and
(70 + 40 + 10) u (1 + |xh|) |w|, dx by half a step and 160 u of the magnitudes that are added.  The sums over rows have at most 256 + M / 148 + 40 steps."""
import itertools

import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
T = {"f": torch.float32, "b": torch.bfloat16}
half = lambda t: torch.finfo(t.dtype).eps / 2  # noqa: E731


def _close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


def _view(g, M, N, t, pad=0, mean=0.0, std=1.0):
    return (torch.randn(M, N + pad, generator=g, device="cuda") * std + mean).to(T[t])[:, :N]


def _hole(M, N, t, pad):
    """an output inside a wider buffer of sevens"""
    whole = torch.full((M + 1, N + pad), 7.0, device="cuda", dtype=T[t])
    return whole, whole[:M, :N]


def _untouched(whole, M, N):
    return bool((whole[M:] == 7).all()) and bool((whole[:, N:] == 7).all())


SIZES = [(1, 1), (5, 1), (1, 8), (3, 7), (300, 9), (5, 64), (257, 96), (700, 40), (2, 4096), (33, 1023), (1501, 1000), (7, 4104), (3, 8191), (2, 16384), (5, 12000), (2, 20001),
         (1, 32768), (400, 2048), (3000, 260)]
MIX = list(itertools.product("fb", ["", "f", "b"], "fb", "fb"))


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("M,N", SIZES)
def test_forward(M, N, layer):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M * 7 + N)
    kind = rr.NORM_LAYER if layer else rr.NORM_RMS
    for i, (xt, ht, yt, wt) in enumerate(MIX[(M + N + layer) % 2::2]):
        pad, eps = (0, 8, 3)[i % 3], (1e-5, 1e-3)[i % 2]
        x = _view(g, M, N, xt, pad, 0.0 if ht else 3.0, 2.0)
        res = _view(g, M, N, ht, pad, 1.0) if ht else None
        w = _view(g, 1, N, wt, mean=1.0)[0].contiguous() if i % 5 else None
        b = _view(g, 1, N, wt)[0].contiguous() if i % 2 else None
        (yw, y), (hw, h) = _hole(M, N, yt, pad), _hole(M, N, ht or "f", pad)
        mean, rstd = (torch.full((M,), 7.0, device="cuda") for _ in range(2))
        out = rr.norm_fwd(x, w, b, residual=res, kind=kind, eps=eps, out=y, h=h if ht else None, mean=mean if layer else None, rstd=rstd)
        assert out is y and _untouched(yw, M, N) and _untouched(hw, M, N)
        stream = x.double() + res.double() if ht else x.double()
        if ht:
            _close(h, stream, (half(h) + U) * stream.abs(), "h")
            stream = h.double()
        want, m, r, xh = ref.norm(stream, w, b, layer, eps)
        size = torch.ones(N, device="cuda", dtype=torch.float64) if w is None else w.double().abs()
        _close(y, want, half(y) * want.abs() + 120 * U * (1 + xh.abs()) * size + 4 * U * (0 if b is None else b.double().abs()), (xt, ht, yt, wt, "y"))
        _close(rstd, r, 40 * U * r, "rstd")
        if layer:
            spread = (stream - m[:, None]).square().mean(1).sqrt()
            _close(mean, m, 2 * U * m.abs() + 70 * U * spread, "mean")
        assert torch.equal(rr.norm_fwd(x, w, b, residual=res, kind=kind, eps=eps, out_dtype=y.dtype), y)  # nothing kept, nothing else differs


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("M,N", SIZES)
def test_backward(M, N, layer):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M * 5 + N)
    kind = rr.NORM_LAYER if layer else rr.NORM_RMS
    ws = rr.alloc_workspace(rr.norm_workspace_bytes(M, N))
    for i, (yt, ht, dt) in enumerate(itertools.product("fb", "fb", "fb")):
        pad = (0, 8, 5)[i % 3]
        dy, h = _view(g, M, N, yt, pad), _view(g, M, N, ht, pad, 1.0, 2.0)
        w = _view(g, 1, N, "bf"[i % 2], mean=1.0)[0].contiguous() if i % 4 else None
        dh = _view(g, M, N, dt, pad) if i % 2 else None
        _, m, r, _ = ref.norm(h, w, None, layer, 1e-5)
        m, r = m.float() if layer else None, r.float()
        whole, dx = _hole(M, N, dt, pad)
        dw, db = (torch.randn(N, generator=g, device="cuda") for _ in range(2))
        old = dw.clone(), db.clone()
        add = i % 3 == 1
        rr.norm_bwd(dy, h, w, m, r, kind=kind, dh=dh, dx=dx, dw=dw, dbias=db, add_dw=add, workspace=ws)
        assert _untouched(whole, M, N)
        want, ww, wb, size, sw, sb = ref.norm_gradients(dy, h, w, m, r, dh)
        _close(dx, want, (half(dx) + U) * want.abs() + 160 * U * size + (0 if dh is None else 2 * U * dh.double().abs()), (yt, ht, dt, "dx"))
        deep = (300 + M / 148) * U
        _close(dw, ww + (old[0].double() if add else 0), deep * sw + 2 * U * (ww.abs() + old[0].double().abs()), "dw")
        _close(db, wb + (old[1].double() if add else 0), deep * sb + 2 * U * (wb.abs() + old[1].double().abs()), "db")
        if not add:  # one at a time, and again: the same bits
            assert torch.equal(rr.norm_bwd(dy, h, w, m, r, kind=kind, dw=torch.empty_like(dw))[1], dw)
            assert torch.equal(rr.norm_bwd(dy, h, w, m, r, kind=kind, dbias=torch.empty_like(db))[2], db)
            assert torch.equal(rr.norm_bwd(dy, h, w, m, r, kind=kind, dh=dh, dx=torch.empty_like(dx))[0], dx)


def test_gradients_against_differences():
    """central differences of the 64-bit forward definition, a few elements each"""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(1)
    M, N, eps = 5, 24, 1e-5
    h, dy, w, b = (torch.randn(*s, generator=g, device="cuda") for s in ((M, N), (M, N), (N,), (N,)))
    for layer in (True, False):
        kind = rr.NORM_LAYER if layer else rr.NORM_RMS
        mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        rr.norm_fwd(h, w, b, kind=kind, eps=eps, mean=mean if layer else None, rstd=rstd)
        dx, dw, db = rr.norm_bwd(dy, h, w, mean if layer else None, rstd, kind=kind, dx=torch.empty_like(h), dw=torch.empty(N, device="cuda"),
                                 dbias=torch.empty(N, device="cuda"))
        loss = lambda h_, w_, b_: float((ref.norm(h_, w_, b_, layer, eps)[0] * dy.double()).sum())  # noqa: E731
        step = 1e-5
        for grad, at in ((dx, 0), (dw, 1), (db, 2)):
            for e in range(0, grad.numel(), 5):
                args = [t.double().clone() for t in (h, w, b)]
                args[at].view(-1)[e] += step
                up = loss(*args)
                args[at].view(-1)[e] -= 2 * step
                # the difference's own error: third derivatives times step^2 and 2^-52 of a loss of about 100 over step
                assert abs((up - loss(*args)) / (2 * step) - float(grad.view(-1)[e])) < 1e-4


def test_in_place():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(2)
    for M, N in ((9, 1023), (300, 512), (4, 9000)):
        x, res, w = _view(g, M, N, "b"), _view(g, M, N, "b"), _view(g, 1, N, "b")[0].contiguous()
        h = torch.empty_like(x)
        want = rr.norm_fwd(x, w, residual=res, h=h, kind=rr.NORM_RMS)
        for k in range(4):
            x2, r2 = x.clone(), res.clone()
            keep = (r2, x2, torch.empty_like(x), torch.empty_like(x))[k]
            y = rr.norm_fwd(x2, w, residual=r2, h=keep, kind=rr.NORM_RMS, out=(x2, r2, x2, r2)[k])
            assert torch.equal(y, want) and torch.equal(keep, h)
        rstd = torch.empty(M, device="cuda")
        rr.norm_fwd(h, w, kind=rr.NORM_RMS, rstd=rstd)
        dy, dh = _view(g, M, N, "b"), _view(g, M, N, "b")
        want = rr.norm_bwd(dy, h, w, None, rstd, kind=rr.NORM_RMS, dh=dh, dx=torch.empty_like(x), dw=torch.empty(N, device="cuda"))
        for k in range(3):
            b = [dy.clone(), h.clone(), dh.clone()]
            got = rr.norm_bwd(b[0], b[1], w, None, rstd, kind=rr.NORM_RMS, dh=b[2], dx=b[k], dw=torch.empty(N, device="cuda"))
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_without_spread_and_far_from_zero():
    import paper_2402_12399_b200 as rr
    N = 4096
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.stack([torch.zeros(N, device="cuda"), torch.full((N,), 1e4, device="cuda"), torch.full((N,), -0.3, device="cuda"),
                     1e4 + torch.randn(N, generator=g, device="cuda"), 1e-20 * torch.randn(N, generator=g, device="cuda"),
                     1e15 * torch.randn(N, generator=g, device="cuda")])
    b = torch.randn(N, generator=g, device="cuda")
    mean, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    y = rr.norm_fwd(x, None, b, mean=mean, rstd=rstd)
    want, m, r, xh = ref.norm(x, None, b, True, 1e-5)
    # rows of one value: the centre is off by less than 70 u |x| in the first look, by 70 u of that in the second: nothing beside the bias
    _close(y, want, 130 * U * (1 + xh.abs()) + 4 * U * b.double().abs(), "y")
    _close(rstd, r, 40 * U * r, "rstd")


def test_a_row_does_not_reach_another():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(4)
    for N in (64, 1023, 4096):
        x = torch.randn(50, N, generator=g, device="cuda")
        clean = rr.norm_fwd(x)
        x[7, N // 2], x[20], x[33, 0] = float("nan"), float("inf"), float("-inf")
        y = rr.norm_fwd(x)
        for i in range(50):
            if i in (7, 20, 33):
                assert torch.isnan(y[i]).any()
            else:
                assert torch.equal(y[i], clean[i])
        rstd = torch.empty(50, device="cuda")
        y = rr.norm_fwd(x, kind=rr.NORM_RMS, rstd=rstd)
        assert torch.isnan(y[7]).all() and torch.isnan(rstd[7])                     # the mean square is not a number
        assert torch.isnan(y[20]).all() and torch.isnan(y[33, 0]) and (y[33, 1:] == 0).all() and (rstd[[20, 33]] == 0).all()    # it is infinite


def test_no_rows():
    import paper_2402_12399_b200 as rr
    x = torch.empty(0, 64, device="cuda")
    assert rr.norm_fwd(x).shape == (0, 64)
    dw, db = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    rr.norm_bwd(x, x, None, x[:, 0], x[:, 0], dx=x.clone(), dw=dw, dbias=db, add_dw=True)
    assert (dw == 1).all() and (db == 1).all()
    rr.norm_bwd(x, x, None, x[:, 0], x[:, 0], dw=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


def test_rows_beyond_32_bits():
    """4.6e9 elements: offsets of 64 bits; the ends are compared"""
    import paper_2402_12399_b200 as rr
    M, N = 140001, 32768
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    x[-3:].normal_()
    rstd = torch.empty(M, device="cuda")
    y = rr.norm_fwd(x, kind=rr.NORM_RMS, rstd=rstd)
    assert torch.equal(y[-3:], rr.norm_fwd(x[-3:].clone(), kind=rr.NORM_RMS)) and (y[:3] == 0).all()
    dx = rr.norm_bwd(y, x, None, None, rstd, kind=rr.NORM_RMS, dx=x)[0]
    assert torch.isfinite(dx[-3:]).all() and (dx[:3] == 0).all()


def test_other_streams_and_graphs():
    import paper_2402_12399_b200 as rr
    M, N = 300, 1024
    x, dy, w = (torch.randn(*s, device="cuda").bfloat16() for s in ((M, N), (M, N), (N,)))
    y, dx, mean, rstd, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty(N, device="cuda")
    ws = rr.alloc_workspace(rr.norm_workspace_bytes(M, N))

    def step():
        rr.norm_fwd(x, w, out=y, mean=mean, rstd=rstd)
        rr.norm_bwd(dy, x, w, mean, rstd, dx=dx, dw=dw, workspace=ws)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    want = [t.clone() for t in (y, dx, dw)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, dx, dw):
        t.fill_(7)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), want))
    x.mul_(2).add_(1)
    graph.replay()
    got = [t.clone() for t in (y, dx, dw)]
    step()
    assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), got)) and not torch.equal(got[0], want[0])


def test_the_binding_refuses():
    import paper_2402_12399_b200 as rr
    x = torch.zeros(4, 8, device="cuda")
    v, m = torch.zeros(8, device="cuda"), torch.zeros(4, device="cuda")
    b = x.bfloat16()
    for bad in (lambda: rr.norm_fwd(x.half()), lambda: rr.norm_fwd(x.t()[:, ::2]), lambda: rr.norm_fwd(x, v[:4]), lambda: rr.norm_fwd(x, v, v.bfloat16()),
                lambda: rr.norm_fwd(x, v.half()), lambda: rr.norm_fwd(x, h=x.clone()), lambda: rr.norm_fwd(x, residual=b, h=x.clone()),
                lambda: rr.norm_fwd(x, residual=b[:3]), lambda: rr.norm_fwd(x, out=torch.empty(4, 7, device="cuda")), lambda: rr.norm_fwd(x, mean=m[:3]),
                lambda: rr.norm_fwd(x, rstd=m.double()), lambda: rr.norm_fwd(x, v.cpu()), lambda: rr.norm_fwd(x, v[::2].repeat(2)[::1][:8][::2]),
                lambda: rr.norm_bwd(x, x, v, m, m, dh=b, dx=x.clone()), lambda: rr.norm_bwd(x, x[:3], v, m, m, dx=x.clone()),
                lambda: rr.norm_bwd(x, x, v, m, m, dw=v.bfloat16()), lambda: rr.norm_bwd(x, x, v, None, m[:2], kind=rr.NORM_RMS, dx=x.clone()),
                lambda: rr.norm_bwd(x, x, v, m, m, dx=x.clone(), workspace=torch.zeros(256, dtype=torch.uint8, device="cuda")),
                lambda: rr.norm_fwd(x, eps=-1.0), lambda: rr.norm_fwd(x, kind=3), lambda: rr.norm_fwd(torch.empty(1, 32769, device="cuda"))):
        with pytest.raises((TypeError, ValueError, rr.RRError)):
            bad()
