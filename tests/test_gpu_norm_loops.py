"""The norm where every block goes round its loop over the rows several times: forward from 32 sets of rows an SM on, backward from one or two on; rows
wider than 4096 columns backward; offsets beyond 2^32 elements; the stored mean of rows far from zero.  Tolerances as where every block takes one set of rows:
u = 2^-24, half a step of the result's type, 120 u (1 + |xh|) |w| for y, 160 u of the magnitudes for dx, at most 300 + M / 148 steps for dw and db."""
import itertools

import pytest
import torch

import step_ref as ref
from test_gpu_norm import MIX, T, U, _close, _hole, _untouched, _view, half

pytestmark = pytest.mark.gpu


# (sets of 64, 4, 1, 1 rows at most: more than 32 * 148 of them in every layout)
@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("M,N", [(320001, 40), (19001, 1000), (5001, 2056), (4801, 4104)])
def test_forward(M, N, layer):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M + N)
    kind = rr.NORM_LAYER if layer else rr.NORM_RMS
    for i, (xt, ht, yt, wt) in enumerate(MIX[layer::2]):
        pad = (0, 8, 3)[i % 3]
        x, res = _view(g, M, N, xt, pad, 0.0 if ht else 3.0, 2.0), _view(g, M, N, ht, pad, 1.0) if ht else None
        w, b = (_view(g, 1, N, wt, mean=1.0)[0].contiguous() for _ in range(2))
        (yw, y), (hw, h) = _hole(M, N, yt, pad), _hole(M, N, ht or "f", pad)
        mean, rstd = (torch.full((M,), 7.0, device="cuda") for _ in range(2))
        rr.norm_fwd(x, w, b, residual=res, kind=kind, out=y, h=h if ht else None, mean=mean if layer else None, rstd=rstd)
        assert _untouched(yw, M, N) and _untouched(hw, M, N)
        stream = x.double()
        if ht:
            stream = stream + res.double()
            _close(h, stream, (half(h) + U) * stream.abs(), "h")
            stream = h.double()
        want, m, r, xh = ref.norm(stream, w, b, layer, 1e-5)
        _close(y, want, half(y) * want.abs() + 120 * U * (1 + xh.abs()) * w.double().abs() + 4 * U * b.double().abs(), (xt, ht, yt, wt, pad, "y"))
        _close(rstd, r, 40 * U * r, "rstd")
        if layer:
            _close(mean, m, 2 * U * m.abs() + 70 * U * (stream - m[:, None]).square().mean(1).sqrt(), "mean")
        if ht:      # the new stream over the old one
            over = torch.empty_like(y)
            rr.norm_fwd(x, w, b, residual=res, kind=kind, out=over, h=res)
            assert torch.equal(res, h) and torch.equal(over, y)


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("M,N", [(1000, 5000), (900, 4104), (700, 9000), (450, 12001), (700, 16392), (450, 20001), (9001, 72)])
def test_backward(M, N, layer):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M + N)
    kind = rr.NORM_LAYER if layer else rr.NORM_RMS
    ws = rr.alloc_workspace(rr.norm_workspace_bytes(M, N))
    for i, (yt, ht, dt) in enumerate(itertools.product("fb", "fb", "fb")):
        pad, through, biased, add = (0, 8, 5)[i % 3], i % 2 == 1, i % 4 < 2, i % 3 == 1
        dy, h = _view(g, M, N, yt, pad), _view(g, M, N, ht, pad, 1.0, 2.0)
        w = _view(g, 1, N, "bf"[i % 2], mean=1.0)[0].contiguous()
        dh = _view(g, M, N, dt, pad) if through else None
        _, m, r, _ = ref.norm(h, w, None, layer, 1e-5)
        m, r = m.float() if layer else None, r.float()
        whole, dx = _hole(M, N, dt, pad)
        dw, db = (torch.randn(N, generator=g, device="cuda") for _ in range(2))
        old = dw.double(), db.double()
        rr.norm_bwd(dy, h, w, m, r, kind=kind, dh=dh, dx=dx, dw=dw, dbias=db if biased else None, add_dw=add, workspace=ws)
        assert _untouched(whole, M, N)
        want, ww, wb, size, sw, sb = ref.norm_gradients(dy, h, w, m, r, dh)
        _close(dx, want, (half(dx) + U) * want.abs() + 160 * U * size + (0 if dh is None else 2 * U * dh.double().abs()), (yt, ht, dt, "dx"))
        deep = (300 + M / 148) * U
        _close(dw, ww + (old[0] if add else 0), deep * sw + 2 * U * (ww.abs() + old[0].abs()), "dw")
        if biased:
            _close(db, wb + (old[1] if add else 0), deep * sb + 2 * U * (wb.abs() + old[1].abs()), "db")
        else:
            assert torch.equal(db.double(), old[1])
        if dh is not None:      # the gradient over the one that came along the stream
            rr.norm_bwd(dy, h, w, m, r, kind=kind, dh=dh, dx=dh, workspace=ws)
            assert torch.equal(dh, dx)


def test_matrices_beyond_32_bits():
    """4.6e9 elements, forward with the new stream over the old one and backward over the stream's gradient; rows at both ends and on both sides of
    elements 2^31 and 2^32 are compared with the same calls on these rows alone (a row's results do not depend on the others)."""
    import paper_2402_12399_b200 as rr
    M, N = 140001, 32768
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = torch.Generator("cuda").manual_seed(1)
    rows = torch.tensor([0, 1, 65535, 65536, 65537, 131071, 131072, 131073, M - 2, M - 1], device="cuda")
    w, b = (torch.randn(N, generator=g, device="cuda").bfloat16() for _ in range(2))
    few_x, few_r = (torch.randn(len(rows), N, generator=g, device="cuda").bfloat16() for _ in range(2))
    few_y, few_m, few_s = torch.empty_like(few_x), *(torch.empty(len(rows), device="cuda") for _ in range(2))
    few_h = few_r.clone()
    rr.norm_fwd(few_x, w, b, residual=few_h, h=few_h, out=few_y, mean=few_m, rstd=few_s)
    x, h, y = (torch.zeros(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    x[rows], h[rows] = few_x, few_r
    rr.norm_fwd(x, w, b, residual=h, h=h, out=y, mean=mean, rstd=rstd)
    assert torch.equal(h[rows], few_h) and torch.equal(y[rows], few_y) and torch.equal(mean[rows], few_m) and torch.equal(rstd[rows], few_s)
    for row in (2, 65534, 65538, 131070, 131074, M - 3):      # rows of zeros: the bias alone
        assert torch.equal(y[row], b) and not h[row].any() and mean[row] == 0
    # backward: y serves as dy, x as the gradient that comes along the stream and is written over
    y.zero_()
    y[rows] = few_y
    dw, db = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    want = rr.norm_bwd(few_y, few_h, w, few_m, few_s, dh=few_x, dx=torch.empty_like(few_x))[0]
    rr.norm_bwd(y, h, w, mean, rstd, dh=x, dx=x, dw=dw, dbias=db)
    assert torch.equal(x[rows], want) and not torch.equal(want, few_x)
    for row in (2, 65534, 65538, 131070, 131074, M - 3):
        assert not x[row].any()
    # the other rows add zeros; ten terms, a rounding each
    _, ww, wb, _, sw, sb = ref.norm_gradients(few_y, few_h, w, few_m, few_s, None)
    _close(dw, ww, 16 * U * sw, "dw")
    _close(db, wb, 16 * U * sb, "db")


@pytest.mark.parametrize("N", [1023, 4096, 9000])
def test_stored_mean_of_rows_far_from_zero(N):
    """The first look at the mean is off by d, at most 70 u of the mean magnitude; where that is more than 4 u of sqrt(var + eps) the second look
    takes it off up to 71 u of the spread and the rounding of the sum.  (Every d below that threshold is itself within 4 u of sqrt(var + eps).)"""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(3)
    z = torch.randn(N, generator=g, device="cuda")
    x = torch.stack([torch.zeros_like(z), torch.full_like(z, 1e4), torch.full_like(z, -0.3), 1e4 + z, -1e6 + z, 300 + 0.01 * z, 1e-20 * z, 1e15 * z])
    mean, rstd = torch.empty(len(x), device="cuda"), torch.empty(len(x), device="cuda")
    rr.norm_fwd(x, mean=mean, rstd=rstd)
    v = x.double()
    m = v.mean(1)
    wide = ((v - m[:, None]).square().mean(1) + 1e-5).sqrt()
    _close(mean, m, 2 * U * m.abs() + 150 * U * torch.minimum(v.abs().mean(1), wide), "mean")
    _close(rstd, 1 / wide, 40 * U / wide, "rstd")
