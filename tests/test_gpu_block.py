"""The operators around the expert layer together with it, as a block of a model uses them in a training step:
projection with activation, dropout and residual -> gate -> routing -> experts -> dropout and residual, the balance and z-loss of a
padded batch, and the way back.  Each piece is compared in 64 bits on the inputs that the GPU handed it; bounds as in the tests of the
layer (2e-2 x RMS, which covers the bf16 roundings between the pieces)."""
import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2402_12399_b200 import synth

pytestmark = pytest.mark.gpu
TOL = 2e-2


def _ratio(got, want, what):
    got, want = (t.double().cpu().numpy() if torch.is_tensor(t) else np.asarray(t, np.float64) for t in (got, want))
    rms = float(np.sqrt((want ** 2).mean()))
    err = float(np.abs(got - want).max())
    assert rms > 0 and err <= TOL * rms, f"{what}: max err {err:.3e} vs rms {rms:.3e}"


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


class Block:
    """Buffers and weights of one block; forward() and backward() make only the library's calls."""

    def __init__(self, S=4, L=512, E=8, k=2, G=4, d=128, d_ff=256, seed=3):
        import helpers
        import paper_2402_12399_b200 as rr
        self.S, self.T, self.E, self.k, self.G, self.d, self.d_ff, self.mode = S, S * L, E, k, G, d, d_ff, 3
        self.C = k * self.T // E
        T = self.T
        self.L = synth.make_layer(T, E, d, d_ff, ("none", 0), seed, "bf16", True, w_std=0.05)
        self.x, self.W1, self.W3, self.W2, self.dy = (helpers.to_torch(v, "bf16") for v in (self.L.hidden, self.L.W1, self.L.W3, self.L.W2, self.L.dout))
        g = torch.Generator("cuda").manual_seed(seed)
        bf = dict(device="cuda", dtype=torch.bfloat16)
        self.Wp = (torch.randn(d, d, generator=g, device="cuda") * d ** -0.5).bfloat16()
        self.bp = (0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16()
        self.Wg = (2 * torch.randn(E, d, generator=g, device="cuda") * d ** -0.5).bfloat16()
        end = torch.tensor([L, L // 3, 0, L - 5], device="cuda")[:S]
        self.live = (torch.arange(L, device="cuda")[None] < end[:, None]).reshape(-1)
        self.p, self.alpha, self.beta, self.scale = 0.1, 1e-2, 1e-3, 30.0
        self.rng_p, self.rng_m = (torch.tensor([17, i], device="cuda") for i in (0, 1))
        self.h, self.z, self.y, self.dmoe = (torch.empty(T, d, **bf) for _ in range(4))
        self.dh16, self.dx, self.dWp, self.dbp = torch.empty(T, d, **bf), torch.empty(T, d, **bf), torch.empty(d, d, device="cuda"), torch.empty(d, device="cuda")
        fb, bb = rr.linear_workspace_bytes(T, d, d)
        self.ws = {n: rr.alloc_workspace(b) for n, b in (("lf", fb), ("lb", bb), ("route", rr.route_workspace_bytes(T, E, k, self.C, G, 3)),
                                                         ("bal", rr.balance_workspace_bytes(T, E, S)), ("gf", rr.gate_workspace_bytes(T, E, d)[0]),
                                                         ("gb", rr.gate_workspace_bytes(T, E, d)[1]))}
        mf, mb, saved = rr.moe_workspace_bytes(T, E, k, self.C, G, d, d_ff, 0, 3)
        self.ws["mf"], self.ws["mb"], self.saved = rr.alloc_workspace(mf), rr.alloc_workspace(mb), torch.empty(saved, dtype=torch.uint8, device="cuda")
        self.tab = rr.alloc_tables(T, E, k, self.C, G, 3)
        self.logits, self.moe = torch.empty(T, E, device="cuda"), torch.empty(T, d, device="cuda")
        self.grads = tuple(torch.empty(*s, device="cuda") for s in ((T, d), (T, E), (E, d_ff, d), (E, d_ff, d), (E, d, d_ff)))
        self.dWg = torch.empty(E, d, device="cuda")

    def forward(self):
        import paper_2402_12399_b200 as rr
        rr.linear_fwd(self.x, self.Wp, self.bp, self.x, act=rr.ACT_SILU, p=self.p, rng=self.rng_p, out=self.h, z=self.z, workspace=self.ws["lf"])
        rr.gate_fwd(self.h, self.Wg, self.logits, self.ws["gf"])
        rr.route(self.logits, self.k, self.C, self.G, self.mode, self.tab, self.ws["route"])
        rr.moe_fwd(self.h, self.W1, self.W3, self.W2, self.logits, self.tab, self.moe, self.saved, self.ws["mf"])
        rr.dropout_fwd(self.moe, self.p, self.rng_m, residual=self.h, out=self.y)
        self.bal = rr.balance_fwd(self.logits, self.tab.topk_expert, self.k, self.alpha, self.beta, segments=self.S, live=self.live, workspace=self.ws["bal"])

    def backward(self):
        import paper_2402_12399_b200 as rr
        dh, dl = self.grads[:2]
        rr.dropout_bwd(self.dy, self.p, self.rng_m, out=self.dmoe)
        rr.moe_bwd(self.dmoe, self.h, self.W1, self.W3, self.W2, self.logits, self.tab, self.saved, workspace=self.ws["mb"], grads=self.grads)
        rr.balance_bwd(self.logits, self.bal[1], self.bal[2], self.k, self.alpha, self.beta, scale=self.scale, live=self.live, dlogits=dl, accumulate=True)
        rr.gate_bwd(dl, self.h, self.Wg, dh, self.dWg, self.ws["gb"])
        rr.dropout_bwd(self.dy, 0.0, None, out=dh, accumulate=True)          # the residual around the experts
        self.dh16.copy_(dh)
        self.dx.copy_(self.dh16)                                              # the residual around the projection
        rr.linear_bwd(self.dh16, self.x, self.Wp, self.z, act=rr.ACT_SILU, p=self.p, rng=self.rng_p, dx=self.dx, dw=self.dWp, dbias=self.dbp,
                      add_dx=True, workspace=self.ws["lb"])

    def outputs(self):
        return [self.h, self.z, self.logits, self.y, *self.bal, self.dmoe, *self.grads, self.dWg, self.dh16, self.dx, self.dWp, self.dbp]

    def check(self):
        import paper_2402_12399_b200 as rr
        for w in self.ws.values():
            rr.check(w)


def test_training_step_of_a_block():
    import helpers
    from oracle import rr_oracle as orc
    b = Block()
    b.forward()
    b.backward()
    b.check()
    z64 = b.x.double() @ b.Wp.double().T + b.bp.double()
    _ratio(b.h, b.x.double() + ref.dropped(ref.act(z64, 4), b.p, b.rng_p), "h")
    a, h = b.logits.cpu().numpy(), _bits(b.h)
    tokens = np.arange(b.T, dtype=np.int32)
    tc = orc.route(a, b.k, b.C, b.G, b.mode)
    helpers.assert_tables_equal(b.tab, tc, "tables")
    moe = orc.forward_tokens(h, b.L.W1, b.L.W3, b.L.W2, a, tc, tokens)
    _ratio(b.y, b.h.double().cpu() + ref.dropped(torch.from_numpy(moe).cuda(), b.p, b.rng_m).cpu(), "y")
    loss, count, n, P, dbal = ref.balance(b.logits, b.tab.topk_expert, b.k, b.alpha, b.beta, b.S, b.live)
    assert torch.equal(b.bal[1].cpu(), count) and torch.equal(b.bal[2].cpu(), n) and int(n[2]) == 0
    assert torch.allclose(b.bal[0].double().cpu(), loss, rtol=1e-5) and torch.allclose(b.bal[3].double().cpu(), P, rtol=1e-5, atol=1e-12)
    # backwards
    dmoe = ref.dropped(b.dy.double(), b.p, b.rng_m)
    _ratio(b.dmoe, dmoe, "gradient of the experts' output")
    want_dh, want_dl = orc.backward_tokens(h, b.L.W1, b.L.W3, b.L.W2, _bits(b.dmoe), a, tc, tokens)
    want_dl = want_dl + b.scale * dbal.numpy()
    want_dWg, gate_dh = orc.gate_bwd(want_dl, h, _bits(b.Wg))
    _ratio(b.grads[1], want_dl, "dlogits")
    _ratio(b.dWg, want_dWg, "dWg")
    want_dh = torch.from_numpy(want_dh + gate_dh).cuda() + b.dy.double()
    _ratio(b.grads[0], want_dh, "dh")
    dz = ref.dropped(b.dh16.double(), b.p, b.rng_p) * ref.act_slope(b.z.double(), 4)
    _ratio(b.dx, b.dh16.double() + dz @ b.Wp.double(), "dx")
    _ratio(b.dWp, dz.T @ b.x.double(), "dWp")
    _ratio(b.dbp, dz.sum(0), "dbp")


def test_captured_step_of_a_block():
    """The whole step in one graph, replayed with other masks and another batch: what the same calls give outside a graph."""
    b = Block()
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward()
        b.backward()
    kept = b.bal
    for i in range(2):
        b.x.copy_(torch.roll(b.x, 77, 0))
        b.rng_p[1:].add_(2), b.rng_m[1:].add_(2)
        b.bal = kept
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in b.outputs()]
        b.forward()
        b.backward()
        torch.cuda.synchronize()
        b.check()
        # (the expert layer adds rows with floating-point atomics: what passes through it agrees to its low bits)
        for i, (x, y) in enumerate(zip(got, b.outputs())):
            assert torch.allclose(x.double(), y.double(), rtol=2e-2, atol=2e-2 * float(y.double().square().mean().sqrt()) + 1e-12), i
        assert torch.equal(got[0], b.h) and torch.equal(got[2], b.logits) and all(torch.equal(x, y) for x, y in zip(got[4:8], b.bal))


def test_masks_of_both_operators_are_the_same():
    """The linear layer's epilogue and the dropout call drop the same elements for the same generator state."""
    import paper_2402_12399_b200 as rr
    for M in (3, 700):
        x, eye = torch.ones(M, 64, device="cuda", dtype=torch.bfloat16), torch.eye(64, device="cuda").bfloat16()
        rng = torch.tensor([5, 6], device="cuda")
        assert torch.equal(rr.linear_fwd(x, eye, p=0.25, rng=rng), rr.dropout_fwd(x, 0.25, rng))


def test_one_workspace_for_every_call_in_turn():
    import paper_2402_12399_b200 as rr
    b = Block()
    b.forward()
    b.backward()
    want = [t.clone() for t in b.outputs()]
    size = max(w.numel() for w in b.ws.values())
    one = rr.alloc_workspace(size)
    b.ws = {n: one for n in b.ws}
    for _ in range(2):
        b.forward()
        b.backward()
    b.check()
    for i, (x, y) in enumerate(zip(want, b.outputs())):
        assert torch.allclose(x.double(), y.double(), rtol=2e-2, atol=2e-2 * float(y.double().square().mean().sqrt()) + 1e-12), i


def test_calls_that_follow_at_once_see_each_other():
    """Every kernel may be made ready while the one in front still runs: chains whose calls read what the call in front wrote and overwrite
    what it read, with and without a synchronisation between the calls."""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(1)
    bf = dict(device="cuda", dtype=torch.bfloat16)
    for M, N in ((700, 512), (5, 4096), (64, 256)):
        w = (torch.randn(N, N, generator=g, device="cuda") * N ** -0.5).bfloat16()
        b = torch.randn(N, generator=g, device="cuda").bfloat16()
        start = torch.randn(M, N, generator=g, device="cuda").bfloat16()
        rng = torch.tensor([3, 0], device="cuda")
        fb, bb = rr.linear_workspace_bytes(M, N, N)
        ws, wb = rr.alloc_workspace(fb), rr.alloc_workspace(bb)

        def chain(wait):
            x, y, z, dw, db = start.clone(), torch.empty(M, N, **bf), torch.empty(M, N, **bf), torch.zeros(N, N, device="cuda"), torch.zeros(N, device="cuda")
            a = torch.empty(M, N, device="cuda")
            for i in range(12):
                for call in (lambda: rr.linear_fwd(x, w, b, x, act=rr.ACT_SILU, p=0.1, rng=rng, out=y, z=z, workspace=ws),
                             lambda: rr.dropout_fwd(y, 0.2, rng, out=x),
                             lambda: rr.dropout_fwd(x, 0.0, None, out=a, out_dtype=torch.float32),
                             lambda: rr.linear_bwd(x, z, w, z, act=rr.ACT_SILU, p=0.1, rng=rng, dx=y, dw=dw, dbias=db, add_dw=True, workspace=wb),
                             lambda: rr.dropout_fwd(y, 0.3, rng, residual=x, out=x)):
                    call()
                    if wait:
                        torch.cuda.synchronize()
                x.clamp_(-4, 4)
            torch.cuda.synchronize()
            rr.check(ws), rr.check(wb)
            return x, y, z, a, dw, db
        for p, q in zip(chain(True), chain(False)):
            assert torch.equal(p, q)


def test_captured_with_branches():
    """A graph whose branches fork and join between the calls gives what the eager calls give."""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(2)
    bf = dict(device="cuda", dtype=torch.bfloat16)
    x, w = torch.randn(300, 256, generator=g, device="cuda").bfloat16(), torch.randn(512, 256, generator=g, device="cuda").bfloat16()
    a, rng = torch.randn(256, 8, generator=g, device="cuda"), torch.tensor([1, 2], device="cuda")
    table = torch.topk(a, 3, 1).indices.int().contiguous()
    ws, ws2, wb = rr.alloc_workspace(256), rr.alloc_workspace(256), rr.alloc_workspace(rr.balance_workspace_bytes(256, 8, 4))
    y = [torch.empty(300, 512, **bf) for _ in range(3)] + [torch.empty(3, 512, **bf)]
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        rr.linear_fwd(x, w, out=y[0], workspace=ws)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            rr.linear_fwd(x, w, act=rr.ACT_GELU, out=y[1], workspace=ws2)
            out = rr.balance_fwd(a, table, 2, 0.1, 0.1, segments=4, workspace=wb)
        rr.dropout_fwd(y[0], 0.5, rng, out=y[2])
        main.wait_stream(side)
        rr.dropout_fwd(y[1], 0.5, rng, residual=y[2], out=y[2])
        rr.linear_fwd(x[:3], w, out=y[3], workspace=ws)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            d = rr.balance_bwd(a, out[1], out[2], 2, 0.1, 0.1)
        main.wait_stream(side)
        return [*y, *out, d]
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in y:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
