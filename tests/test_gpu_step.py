"""Embedding, norms and clip together with the expert layer, as a training step uses them: ids -> embedding -> norm -> gate, routing, experts ->
residual add and norm -> projection, the way back, and the clip of all gradients.  Every piece is compared in 64 bits on the inputs that the
GPU handed it, within the roundings that the tests of the single operators derive; what passes through the experts within 2e-2 x RMS, as in
their own tests."""
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist())


class Step:
    """Buffers and weights; forward() and backward() make only the library's calls."""

    def __init__(self, S=4, L=256, V=500, E=8, k=2, G=4, d=128, d_ff=256, seed=5):
        import paper_2402_12399_b200 as rr
        g = torch.Generator("cuda").manual_seed(seed)
        T = self.T = S * L
        self.E, self.k, self.G, self.C, self.V, self.scale, self.bound = E, k, G, k * T // E, V, d ** 0.5, 0.5
        bf, f32 = dict(device="cuda", dtype=torch.bfloat16), dict(device="cuda", dtype=torch.float32)

        def normal(*shape, std=1.0):
            return (std * torch.randn(*shape, generator=g, device="cuda")).bfloat16()
        self.table, self.Wg, self.W1, self.W3, self.W2 = normal(V, d, std=d ** -0.5), normal(E, d, std=0.2), *(normal(E, d_ff, d, std=0.05) for _ in range(2)), normal(E, d, d_ff, std=0.05)
        self.Wp, self.w1, self.w2, self.b2, self.dy = normal(d, d, std=d ** -0.5), 1 + normal(d, std=0.1), 1 + normal(d, std=0.1), normal(d, std=0.1), normal(T, d)
        ids = torch.randint(0, V, (S, L), generator=g, device="cuda")
        ids = torch.where(torch.rand(S, L, generator=g, device="cuda") < 0.2, torch.full_like(ids, 7), ids)
        end = torch.tensor([L, L // 3, 1, L - 5], device="cuda")[:S]
        self.ids = torch.where(torch.arange(L, device="cuda")[None] < end[:, None], ids, torch.full_like(ids, -1))
        self.x0, self.n1, self.h1, self.n2, self.y, self.dh1, self.dx0 = (torch.empty(T, d, **bf) for _ in range(7))
        self.r1, self.r2, self.m2, self.moe, self.dn2 = torch.empty(T, **f32), torch.empty(T, **f32), torch.empty(T, **f32), torch.empty(T, d, **f32), torch.empty(T, d, **f32)
        self.logits = torch.empty(T, E, **f32)
        self.moe_grads = tuple(torch.empty(*s, **f32) for s in ((T, d), (T, E), (E, d_ff, d), (E, d_ff, d), (E, d, d_ff)))
        self.dtable, self.dWg, self.dw1, self.dw2, self.db2 = torch.empty(V, d, **f32), torch.empty(E, d, **f32), torch.empty(d, **f32), torch.empty(d, **f32), torch.empty(d, **f32)
        self.dWp = torch.empty(d, d, **bf)
        self.clipped = [self.dtable, self.dw1, self.dWg, *self.moe_grads[2:], self.dw2, self.db2, self.dWp]
        self.norm = torch.empty(2, **f32)
        self.tab = rr.alloc_tables(T, E, k, self.C, G, 3)
        mf, mb, saved = rr.moe_workspace_bytes(T, E, k, self.C, G, d, d_ff, 0, 3)
        self.saved = torch.empty(saved, dtype=torch.uint8, device="cuda")
        self.ws = {n: rr.alloc_workspace(b) for n, b in (("ef", 256), ("eb", rr.embed_workspace_bytes(T, V, d)[1]), ("nb", rr.norm_workspace_bytes(T, d)),
                                                         ("lf", rr.linear_workspace_bytes(T, d, d)[0]), ("lb", rr.linear_workspace_bytes(T, d, d)[1]),
                                                         ("route", rr.route_workspace_bytes(T, E, k, self.C, G, 3)), ("gf", rr.gate_workspace_bytes(T, E, d)[0]),
                                                         ("gb", rr.gate_workspace_bytes(T, E, d)[1]), ("mf", mf), ("mb", mb), ("clip", rr.clip_workspace_bytes()))}
        self.plan = rr.grad_plan(self.clipped)

    def forward(self):
        import paper_2402_12399_b200 as rr
        w = self.ws
        rr.embed_fwd(self.ids, self.table, scale=self.scale, out=self.x0, workspace=w["ef"])
        rr.norm_fwd(self.x0, self.w1, kind=rr.NORM_RMS, out=self.n1, rstd=self.r1)
        rr.gate_fwd(self.n1, self.Wg, self.logits, w["gf"])
        rr.route(self.logits, self.k, self.C, self.G, 3, self.tab, w["route"])
        rr.moe_fwd(self.n1, self.W1, self.W3, self.W2, self.logits, self.tab, self.moe, self.saved, w["mf"])
        rr.norm_fwd(self.moe, self.w2, self.b2, residual=self.x0, h=self.h1, out=self.n2, mean=self.m2, rstd=self.r2)
        rr.linear_fwd(self.n2, self.Wp, out=self.y, workspace=w["lf"])

    def backward(self):
        import paper_2402_12399_b200 as rr
        w = self.ws
        rr.linear_bwd(self.dy, self.n2, self.Wp, dx=self.dn2, dw=self.dWp, workspace=w["lb"])
        rr.norm_bwd(self.dn2, self.h1, self.w2, self.m2, self.r2, dx=self.dh1, dw=self.dw2, dbias=self.db2, workspace=w["nb"])
        rr.moe_bwd(self.dh1, self.n1, self.W1, self.W3, self.W2, self.logits, self.tab, self.saved, workspace=w["mb"], grads=self.moe_grads)
        rr.gate_bwd(self.moe_grads[1], self.n1, self.Wg, self.moe_grads[0], self.dWg, w["gb"])
        rr.norm_bwd(self.moe_grads[0], self.x0, self.w1, None, self.r1, kind=rr.NORM_RMS, dh=self.dh1, dx=self.dx0, dw=self.dw1, workspace=w["nb"])
        rr.embed_bwd(self.ids, self.dx0, self.dtable, scale=self.scale, workspace=w["eb"])

    def clip(self):
        import paper_2402_12399_b200 as rr
        rr.clip_grads(self.plan, self.bound, norm=self.norm, workspace=self.ws["clip"])

    def outputs(self):
        return [self.x0, self.n1, self.logits, self.moe, self.h1, self.n2, self.y, self.dn2, self.dh1, *self.moe_grads[:2], self.dx0, self.norm, *self.clipped]

    def check(self):
        import paper_2402_12399_b200 as rr
        for w in self.ws.values():
            rr.check(w)


def test_training_step():
    s = Step()
    s.forward()
    s.backward()
    s.check()
    before = [t.clone() for t in s.clipped]
    s.clip()
    s.check()
    ids = s.ids.view(-1)
    half = 2.0 ** -8
    want = ref.embed(ids, s.table, float(torch.tensor(s.scale)))
    _close(s.x0, want, (half + U) * want.abs(), "x0")
    assert (s.x0[ids < 0] == 0).all() and (ids < 0).any()
    y, _, r, xh = ref.norm(s.x0, s.w1, None, False, 1e-5)
    _close(s.n1, y, half * y.abs() + 120 * U * (1 + xh.abs()) * s.w1.double().abs(), "n1")
    _close(s.r1, r, 40 * U * r, "r1")
    h = s.moe.double() + s.x0.double()
    _close(s.h1, h, (half + U) * h.abs(), "h1")
    y, m, r, xh = ref.norm(s.h1, s.w2, s.b2, True, 1e-5)
    _close(s.n2, y, half * y.abs() + 120 * U * (1 + xh.abs()) * s.w2.double().abs() + 4 * U * s.b2.double().abs(), "n2")
    # backwards (the sums over rows have at most 256 + T / 148 + 40 steps)
    deep = (300 + s.T / 148) * U
    dx, dw, db, size, sw, sb = ref.norm_gradients(s.dn2, s.h1, s.w2, s.m2, s.r2, None)
    _close(s.dh1, dx, (half + U) * dx.abs() + 160 * U * size, "dh1")
    by = {id(t): b for t, b in zip(s.clipped, before)}
    _close(by[id(s.dw2)], dw, deep * sw, "dw2")
    _close(by[id(s.db2)], db, deep * sb, "db2")
    dx, dw, _, size, sw, _ = ref.norm_gradients(s.moe_grads[0], s.x0, s.w1, None, s.r1, s.dh1)
    _close(s.dx0, dx, (half + U) * dx.abs() + 160 * U * size + 2 * U * s.dh1.double().abs(), "dx0")
    _close(by[id(s.dw1)], dw, deep * sw, "dw1")
    want, size = ref.embed_gradient(ids, s.dx0, s.V, float(torch.tensor(s.scale)))
    _close(by[id(s.dtable)], want, (48 + s.T / 64) * U * size, "dtable")
    n, f = ref.clip(before, s.bound)
    assert abs(float(s.norm[0]) - n) <= 6 * U * n and abs(float(s.norm[1]) - f) <= 6 * U * f and f < 1
    for t, b in zip(s.clipped, before):
        want = b.double() * f
        _close(t, want, torch.finfo(t.dtype).eps / 2 * want.abs() + 8 * U * want.abs(), "clipped")


def test_captured_step():
    """The whole step in one graph, replayed with other tokens: what the same calls give outside a graph."""
    s = Step()
    for part in (s.forward, s.backward, s.clip):
        part()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for part in (s.forward, s.backward, s.clip):
            part()
    for _ in range(2):
        s.ids.copy_(torch.roll(s.ids.view(-1), 77).view(s.ids.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in s.outputs()]
        for part in (s.forward, s.backward, s.clip):
            part()
        s.check()
        # (the expert layer adds rows with floating-point atomics: what passes through it agrees to its low bits)
        for i, (x, y) in enumerate(zip(got, s.outputs())):
            assert torch.allclose(x.double(), y.double(), rtol=2e-2, atol=2e-2 * float(y.double().square().mean().sqrt()) + 1e-12), i
        assert all(torch.equal(x, y) for x, y in zip(got[:3], s.outputs()))


def test_one_workspace_for_every_call_in_turn():
    import paper_2402_12399_b200 as rr
    s = Step()
    for part in (s.forward, s.backward, s.clip):
        part()
    want = [t.clone() for t in s.outputs()]
    one = rr.alloc_workspace(max(w.numel() for w in s.ws.values()))
    s.ws = {n: one for n in s.ws}
    for _ in range(2):
        for part in (s.forward, s.backward, s.clip):
            part()
    s.check()
    for i, (x, y) in enumerate(zip(want, s.outputs())):
        assert torch.allclose(x.double(), y.double(), rtol=2e-2, atol=2e-2 * float(y.double().square().mean().sqrt()) + 1e-12), i


def test_calls_that_follow_at_once_see_each_other():
    """Every kernel may be made ready while the one in front still runs: a chain whose calls read what the call in front wrote and overwrite what
    it read, with and without a synchronisation between the calls."""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(1)
    for n, V, d in ((300, 40, 256), (5000, 900, 64), (3, 7, 4096), (700, 100, 1023)):
        ids = torch.randint(-1, V, (n,), generator=g, device="cuda")
        start, w = torch.randn(V, d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda").bfloat16()
        we, wn, wc = rr.alloc_workspace(rr.embed_workspace_bytes(n, V, d)[1]), rr.alloc_workspace(rr.norm_workspace_bytes(n, d)), rr.alloc_workspace(rr.clip_workspace_bytes())

        def chain(wait):
            table, x, y, rstd, dw, norm = start.clone(), torch.empty(n, d, device="cuda"), torch.empty(n, d, device="cuda"), torch.empty(n, device="cuda"), torch.empty(d, device="cuda"), torch.empty(2, device="cuda")
            plan = rr.grad_plan([table, dw])
            for i in range(8):
                for call in (lambda: rr.embed_fwd(ids, table, out=x, workspace=we), lambda: rr.norm_fwd(x, w, residual=x, h=x, kind=rr.NORM_RMS, out=y, rstd=rstd),
                             lambda: rr.norm_bwd(y, x, w, None, rstd, kind=rr.NORM_RMS, dh=y, dx=x, dw=dw, workspace=wn),
                             lambda: rr.embed_bwd(ids, x, table, scale=0.5, accumulate=i % 2 == 1, workspace=we), lambda: rr.clip_grads(plan, 3.0, norm=norm, workspace=wc)):
                    call()
                    if wait:
                        torch.cuda.synchronize()
            torch.cuda.synchronize()
            for ws in (we, wn, wc):
                rr.check(ws)
            return table, x, y, rstd, dw, norm
        for p, q in zip(chain(True), chain(False)):
            assert torch.equal(p, q) and torch.isfinite(p).all()
