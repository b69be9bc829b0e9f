"""rr_linear_fwd / rr_linear_bwd against the 64-bit statement, element by element.

Two kinds of inputs.  Small whole numbers: every product and sum is a whole number below 2^24, the tensor cores and the
fp32 epilogue compute it without rounding (a dropout of 1/2 multiplies by 2), so fp32 results have to be EQUAL and bf16
ones equal to one rounding: a misplaced row, column, k-block or mask bit cannot hide.  Normal deviates: the bound per
element is the sum of
  - the rounding to the result's type: eps/2 of the value (twice where a bf16 value is rounded on the way);
  - the tensor cores' adder, documented as n/16 * 2^-23 of the sum of the magnitudes of the n products, plus 8 steps of fp32;
  - the activation: 3e-6 (1 + |z|) absolute, and its slope (at most 1.13) times the error of z;
  - backward: dz is rounded to bf16, so each product of the contraction may be off by 2^-8 of itself."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8       # half a step of bf16, relative
# (the long ones: few tiles and a long contraction, which the backward pass splits)
LONG = [(4099, 136, 264), (9001, 264, 520), (300, 4104, 264), (20011, 24, 8)]
SIZES = [(1, 8, 8), (2, 64, 64), (31, 136, 72), (33, 72, 136), (64, 1032, 8), (127, 8, 520), (129, 264, 520), (255, 520, 264), (257, 512, 1032), (700, 648, 392)]


def _rng(seed, offset=3):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def _ints(g, *shape, most=3):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").bfloat16()


def _view(t, pad):
    """the same matrix with `pad` more columns between its rows"""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _adder(n, magnitudes):
    return (n / 16 + 8) * 2.0 ** -23 * magnitudes


def _assert_within(got, want, tol, what=""):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


@pytest.mark.parametrize("M,N,K", SIZES + LONG)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_whole_numbers_are_exact(M, N, K, dtype):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M + N)
    x, w, b = _ints(g, M, K), _ints(g, N, K), _ints(g, N, most=9)
    r = _ints(g, M, N, most=9).to(dtype)
    rng = _rng(M)
    exact = x.double() @ w.double().T
    y = rr.linear_fwd(x, w, out_dtype=dtype)
    rr.check(y._workspace)
    assert torch.equal(y, exact.to(dtype))
    z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    y = rr.linear_fwd(x, w, b, r, act=rr.ACT_RELU, p=0.5, rng=rng, out_dtype=dtype, z=z)
    assert torch.equal(z, (exact + b.double()).to(torch.bfloat16))
    assert torch.equal(y, (r.double() + ref.dropped((exact + b.double()).clamp(min=0), 0.5, rng)).to(dtype))
    # gradients: dz = 2 keep dy [z > 0]
    dy, zz = _ints(g, M, N), _ints(g, M, N)
    dz = ref.dropped(dy.double(), 0.5, rng) * (zz.double() > 0)
    dx, dw = torch.empty(M, K, dtype=dtype, device="cuda"), torch.empty(N, K, dtype=dtype, device="cuda")
    db = torch.empty(N, device="cuda")
    rr.linear_bwd(dy, x, w, zz, act=rr.ACT_RELU, p=0.5, rng=rng, dx=dx, dw=dw, dbias=db)
    rr.check(dx._workspace)
    want = (dz @ w.double(), dz.T @ x.double(), dz.sum(0))
    assert torch.equal(dx, want[0].to(dtype)) and torch.equal(dw, want[1].to(dtype)) and torch.equal(db, want[2].float())
    if dtype == torch.float32:                                 # added to what is there
        rr.linear_bwd(dy, x, w, zz, act=rr.ACT_RELU, p=0.5, rng=rng, dx=dx, dw=dw, dbias=db, add_dx=True, add_dw=True)
        assert torch.equal(dx, 2 * want[0].float()) and torch.equal(dw, 2 * want[1].float()) and torch.equal(db, 2 * want[2].float())


@pytest.mark.parametrize("M,N,K", SIZES + [(1, 1032, 2056), (5, 4096, 1024), (48, 1032, 2056), (300, 2048, 4104), (1111, 1416, 968)])
@pytest.mark.parametrize("act", range(5))
def test_forward(M, N, K, act):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M * 7 + act)
    pad = (0, 8, 24)[(M + act) % 3]
    x = _view(torch.randn(M, K, generator=g, device="cuda").bfloat16(), pad)
    w = (torch.randn(N, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    b = torch.randn(N, generator=g, device="cuda").bfloat16()
    for dtype, p, with_b, with_r in ((torch.bfloat16, 0.1, True, True), (torch.bfloat16, 0.0, False, False), (torch.float32, 0.3, True, True)):
        r = _view(torch.randn(M, N, generator=g, device="cuda").to(dtype), pad) if with_r else None
        rng = _rng(N + act, 1 << 40) if p else None
        z = _view(torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), pad)
        wide = torch.full((M, N + pad), 5.0, dtype=dtype, device="cuda")
        y = rr.linear_fwd(x, w, b if with_b else None, r, act=act, p=p, rng=rng, out=wide[:, :N], z=z)
        rr.check(y._workspace)
        assert torch.all(wide[:, N:] == 5.0)                   # what lies between the rows stays
        z64 = x.double() @ w.double().T + (b.double() if with_b else 0)
        mag = x.double().abs() @ w.double().abs().T + (b.double().abs() if with_b else 0)
        _assert_within(z, z64, HALF * z64.abs() + 2 * _adder(K, mag), "z")
        v = ref.act(z64, act)
        keep = ref.dropped(torch.ones_like(v), p, rng)         # 0 or the factor
        want = v * keep + (r.double() if with_r else 0)
        tol = torch.finfo(dtype).eps / 2 * want.abs() + keep * (1.2 * _adder(K, mag) + 3e-6 * (1 + z64.abs())) * 1.01 + 2.0 ** -22 * want.abs()
        _assert_within(y, want, tol, "y")


@pytest.mark.parametrize("M,N,K", SIZES + [(3, 1032, 2056), (300, 2048, 1032), (1111, 1416, 968)] + LONG)
@pytest.mark.parametrize("act", range(5))
def test_gradients(M, N, K, act):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M * 5 + act)
    pad = (0, 8, 24)[(M + act) % 3]
    x = _view(torch.randn(M, K, generator=g, device="cuda").bfloat16(), pad)
    w = (torch.randn(N, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    dy = _view(torch.randn(M, N, generator=g, device="cuda").bfloat16(), pad)
    z = _view((1.5 * torch.randn(M, N, generator=g, device="cuda")).bfloat16(), pad) if act else None
    for dtype, p in ((torch.bfloat16, 0.1), (torch.float32, 0.0)):
        rng = _rng(K + act) if p else None
        dx = _view(torch.empty(M, K, dtype=dtype, device="cuda"), pad)
        dw, db = torch.empty(N, K, dtype=dtype, device="cuda"), torch.empty(N, device="cuda")
        rr.linear_bwd(dy, x, w, z, act=act, p=p, rng=rng, dx=dx, dw=dw, dbias=db)
        rr.check(dx._workspace)
        dz = ref.dropped(dy.double(), p, rng) * (ref.act_slope(z.double(), act) if act else 1)
        err = (HALF if act else 0) * 1.01 * dz.abs() + 4e-6 * dy.double().abs() / (1 - p) * (1 + (z.double().abs() if act else 0)) * bool(act)
        for got, want, mag, bound, n in ((dx, dz @ w.double(), dz.abs() @ w.double().abs(), err @ w.double().abs(), N),
                                         (dw, dz.T @ x.double(), dz.abs().T @ x.double().abs(), err.T @ x.double().abs(), M)):
            _assert_within(got, want, torch.finfo(dtype).eps / 2 * want.abs() + bound + _adder(n, mag) + 2.0 ** -22 * want.abs(), "product")
        exact_err = 4e-6 * (dy.double().abs() / (1 - p) * (1 + (z.double().abs() if act else 0))).sum(0) + (M / 8 + 16) * 2.0 ** -24 * dz.abs().sum(0)
        _assert_within(db, dz.sum(0), exact_err, "dbias")


def test_gradients_are_the_derivatives_of_the_forward_pass():
    """Central differences of sum(dy * y) in 64 bits at points of a small layer, mask included, against the kernel's gradients."""
    import paper_2402_12399_b200 as rr
    M, N, K, p = 9, 24, 16, 0.25
    g = torch.Generator("cuda").manual_seed(2)
    x, w = torch.randn(M, K, generator=g, device="cuda").bfloat16(), (torch.randn(N, K, generator=g, device="cuda") * 0.5).bfloat16()
    b, dy = torch.randn(N, generator=g, device="cuda").bfloat16(), torch.randn(M, N, generator=g, device="cuda").bfloat16()
    rng = _rng(6)
    for act in range(5):
        def loss(x64, w64, b64):
            return (dy.double() * ref.dropped(ref.act(x64 @ w64.T + b64, act), p, rng)).sum()
        z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        rr.linear_fwd(x, w, b, act=act, p=p, rng=rng, z=z)
        dx, dw, db = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
        rr.linear_bwd(dy, x, w, z, act=act, p=p, rng=rng, dx=dx, dw=dw, dbias=db)
        at = [x.double(), w.double(), b.double()]
        for which, (got, i) in enumerate(((dx, (4, 7)), (dw, (11, 3)), (db, (5,)))):
            h = 1e-5
            up, down = [t.clone() for t in at], [t.clone() for t in at]
            up[which][i] += h
            down[which][i] -= h
            diff = float(loss(*up) - loss(*down)) / (2 * h)
            # z and dz are rounded to bf16: each of up to 24 terms is off by 2^-8 (dz) + 2^-8 |z| |act''| / |act'| (below 2^-6 in all)
            scale = float((dy.double().abs()).max()) * 4 * 24 * 2.0 ** -6
            assert abs(float(got[i]) - diff) <= scale, (act, which, float(got[i]), diff)


def test_rows_of_infinities_and_nans_stay_in_their_rows():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(1)
    x, w = _ints(g, 300, 72), _ints(g, 136, 72)
    want = [rr.linear_fwd(x, w, act=a) for a in range(5)]
    x2 = x.clone()
    x2[7], x2[299] = float("nan"), float("inf")
    for a in range(5):
        y = rr.linear_fwd(x2, w, act=a)
        same = torch.ones(300, dtype=torch.bool)
        same[[7, 299]] = False
        assert torch.equal(y[same], want[a][same]) and torch.isnan(y[7]).all()
    far = torch.tensor([[100.0], [-100.0], [3e38], [-3e38]], device="cuda").bfloat16()
    eye = torch.zeros(8, 8, device="cuda", dtype=torch.bfloat16)
    eye[:, 0] = 1
    x = torch.zeros(4, 8, device="cuda", dtype=torch.bfloat16)
    x[:, :1] = far
    for a in range(1, 5):                                      # the limits of the activations and of their slopes
        y = rr.linear_fwd(x, eye, act=a)
        assert torch.equal(y, far.clamp(min=0).expand(4, 8))
        dx = torch.empty(4, 8, device="cuda")
        rr.linear_bwd(torch.ones_like(y), x, eye, y * 0 + far, act=a, dx=dx)
        assert torch.equal(dx[:, 0], torch.tensor([8.0, 0.0, 8.0, 0.0], device="cuda"))


@pytest.mark.parametrize("M", [5, 333])
def test_in_place_residual_and_parts_of_the_gradient(M):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(4)
    x, w, b = _ints(g, M, 200), _ints(g, 520, 200), _ints(g, 520)
    for dtype in (torch.bfloat16, torch.float32):
        r = _ints(g, M, 520).to(dtype)
        want = rr.linear_fwd(x, w, b, r, act=rr.ACT_SILU)
        same = r.clone()
        assert rr.linear_fwd(x, w, b, same, act=rr.ACT_SILU, out=same) is same and torch.equal(same, want)
    dy = _ints(g, M, 520)
    bufs = [torch.empty(M, 200, device="cuda"), torch.empty(520, 200, device="cuda"), torch.empty(520, device="cuda")]
    rr.linear_bwd(dy, x, w, dx=bufs[0], dw=bufs[1], dbias=bufs[2])
    for keep in ((0,), (1,), (2,), (0, 2), (1, 2), ()):
        part = [torch.full_like(t, 3.0) if i in keep else None for i, t in enumerate(bufs)]
        rr.linear_bwd(dy, x if 1 in keep else None, w, dx=part[0], dw=part[1], dbias=part[2])
        assert all(torch.equal(part[i], bufs[i]) for i in keep)


def test_everything_dropped():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(4)
    for M in (3, 300):
        x, w, r, rng = _ints(g, M, 64), _ints(g, 72, 64), _ints(g, M, 72), _rng(1)
        x[0] = float("nan")
        assert torch.equal(rr.linear_fwd(x, w, residual=r, act=rr.ACT_GELU, p=1.0, rng=rng), r)
        dx, dw, db = torch.ones(M, 64, device="cuda"), torch.ones(72, 64, device="cuda"), torch.ones(72, device="cuda")
        x[0] = 1
        rr.linear_bwd(r, x, w, p=1.0, rng=rng, dx=dx, dw=dw, dbias=db)
        assert not dx.any() and not dw.any() and not db.any()


def test_no_tokens():
    import paper_2402_12399_b200 as rr
    x, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(8, 64, dtype=torch.bfloat16, device="cuda")
    assert rr.linear_fwd(x, w).shape == (0, 8)
    for add in (False, True):
        dw, db = torch.ones(8, 64, device="cuda"), torch.ones(8, device="cuda")
        rr.linear_bwd(torch.empty(0, 8, dtype=torch.bfloat16, device="cuda"), x, w, dx=torch.empty(0, 64, device="cuda"), dw=dw, dbias=db, add_dw=add)
        assert torch.all(dw == float(add)) and torch.all(db == float(add))


def test_repeats_and_streams():
    """Bit for bit the same, twice and on two streams at once with a workspace each."""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(4)
    x, w = torch.randn(1500, 1024, generator=g, device="cuda").bfloat16(), torch.randn(1416, 1024, generator=g, device="cuda").bfloat16()
    dy, z = torch.randn(1500, 1416, generator=g, device="cuda").bfloat16(), torch.randn(1500, 1416, generator=g, device="cuda").bfloat16()
    rng = _rng(5)

    def once():
        out = [rr.linear_fwd(x, w, act=2, p=0.1, rng=rng), rr.linear_fwd(x[:3], w, act=2, p=0.1, rng=rng)]
        grads = [torch.empty(1500, 1024, device="cuda"), torch.empty(1416, 1024, device="cuda"), torch.empty(1416, device="cuda")]
        rr.linear_bwd(dy, x, w, z, act=2, p=0.1, rng=rng, dx=grads[0], dw=grads[1], dbias=grads[2])
        return out + grads
    want = once()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(once())
    torch.cuda.synchronize()
    for o in got:
        assert all(torch.equal(a, b) for a, b in zip(o, want))


def test_captured_step_takes_new_inputs_and_masks():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(4)
    x, w = _ints(g, 100, 264), _ints(g, 136, 264)
    dy, z, y = _ints(g, 100, 136), torch.empty(100, 136, dtype=torch.bfloat16, device="cuda"), torch.empty(100, 136, device="cuda")
    dx, dw, db = torch.empty(100, 264, device="cuda"), torch.empty(136, 264, device="cuda"), torch.empty(136, device="cuda")
    rng = _rng(5)
    fb, bb = rr.linear_workspace_bytes(100, 136, 264)
    ws_f, ws_b = rr.alloc_workspace(fb), rr.alloc_workspace(bb)

    def step():
        rr.linear_fwd(x, w, act=1, p=0.5, rng=rng, out=y, z=z, workspace=ws_f)
        rr.linear_bwd(dy, x, w, z, act=1, p=0.5, rng=rng, dx=dx, dw=dw, dbias=db, workspace=ws_b)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        rng[1:].add_(1)
    for _ in range(3):
        x.copy_(_ints(g, 100, 264))
        pre = x.double() @ w.double().T
        want = ref.dropped(pre.clamp(min=0), 0.5, rng)
        dz = ref.dropped(dy.double(), 0.5, rng) * (pre > 0)
        graph.replay()
        torch.cuda.synchronize()
        rr.check(ws_f), rr.check(ws_b)
        assert torch.equal(y, want.float()) and torch.equal(dx, (dz @ w.double()).float()) and torch.equal(dw, (dz.T @ x.double()).float())
        assert torch.equal(db, dz.sum(0).float())


def test_results_behind_32_bits():
    """y of 2^32 + elements and more: 64-bit offsets and the mask's counter; the last rows against the first ones' arithmetic."""
    import paper_2402_12399_b200 as rr
    M, N, K = 262400, 16392, 8
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    g = torch.Generator("cuda").manual_seed(4)
    x, w, rng = _ints(g, M, K), _ints(g, N, K), _rng(5)
    y = rr.linear_fwd(x, w, p=0.5, rng=rng)
    rr.check(y._workspace)
    for r0 in (0, 131072, M - 3):
        want = x[r0:r0 + 3].double() @ w.double().T
        keep, _ = ref.keep_mask(5, 3, r0 * N, 3 * N, 0.5)
        want = torch.where(torch.from_numpy(keep).cuda().view(3, N), 2 * want, torch.zeros_like(want))
        assert torch.equal(y[r0:r0 + 3], want.bfloat16())


def test_binding_refuses():
    import paper_2402_12399_b200 as rr
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w, dy, rng = torch.zeros(16, 64, **bf), torch.zeros(24, 64, **bf), torch.zeros(16, 24, **bf), _rng(1)
    dx = torch.zeros(16, 64, **bf)
    for call, err in [(lambda: rr.linear_fwd(x.float(), w), TypeError), (lambda: rr.linear_fwd(x, w.float()), TypeError),
                      (lambda: rr.linear_fwd(x[:, :32], w), ValueError), (lambda: rr.linear_fwd(x, w, w[0]), ValueError),
                      (lambda: rr.linear_fwd(x, w, residual=dy[:8]), ValueError), (lambda: rr.linear_fwd(x, w, p=0.5), ValueError),
                      (lambda: rr.linear_fwd(x, w, p=1.5, rng=rng), rr.RRError), (lambda: rr.linear_fwd(x, w, act=5), rr.RRError),
                      (lambda: rr.linear_fwd(x[:, :12].contiguous(), w[:, :12].contiguous()), rr.RRError),     # K not a multiple of 8
                      (lambda: rr.linear_fwd(x, w[:20]), rr.RRError),                                          # N not a multiple of 8
                      (lambda: rr.linear_fwd(torch.zeros(64, 16, **bf).T, w), ValueError),                     # column-major
                      (lambda: rr.linear_fwd(torch.zeros(1, 64, **bf).expand(16, 64), w), ValueError),         # rows lie over each other
                      (lambda: rr.linear_fwd(torch.zeros(16, 68, **bf)[:, :64], w), rr.RRError),               # rows not 16-byte aligned
                      (lambda: rr.linear_fwd(torch.zeros(16 * 64 + 1, **bf)[1:].view(16, 64), w), rr.RRError),
                      (lambda: rr.linear_fwd(x.cpu(), w), ValueError), (lambda: rr.linear_fwd(x, w, residual=dy.float(), out=dy), TypeError),
                      (lambda: rr.linear_fwd(x, w, workspace=torch.zeros(128, dtype=torch.uint8, device="cuda")), rr.RRError),
                      (lambda: rr.linear_bwd(dy, x, w, act=2, dx=dx), rr.RRError),                             # the pre-activations are missing
                      (lambda: rr.linear_bwd(dy, None, w, dw=torch.zeros(24, 64, **bf)), rr.RRError),
                      (lambda: rr.linear_bwd(dy, x, w, dbias=torch.zeros(24, **bf)), TypeError),
                      (lambda: rr.linear_bwd(dy, x, w, dw=torch.zeros(24, 32, **bf)), ValueError)]:
        with pytest.raises(err):
            call()
