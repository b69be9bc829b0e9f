"""The products inside the training step that the embedding, the norms and the clip are part of: gate, projection and their gradients against
64-bit products of the inputs that the GPU handed them, the expert layer and its gradients against the oracle.

Products: the tensor cores' adder is off by n / 16 2^-23 of the magnitudes of n products and 8 steps of fp32, and the result by half a step of its type; the
gate's gradients by 1e-4 x RMS (sums in fp32 in some order of T or E terms), the expert layer's result and the gradients of its
input and logits by 2e-2 x RMS, as in their own tests; its weights' gradients by what the rounding of their operands allows."""
import numpy as np
import pytest
import torch

import step_ref as ref
from test_gpu_step import U, Step, _close

pytestmark = pytest.mark.gpu


def _adder(n, size):
    return (n / 16 + 8) * 2.0 ** -23 * size


def _product(got, a, b, what):
    """got = a b, in its type"""
    a, b = a.double(), b.double()
    want = a @ b
    _close(got, want, torch.finfo(got.dtype).eps / 2 * want.abs() + _adder(a.shape[1], a.abs() @ b.abs()), what)


def _rms(got, want, tol, what):
    err, rms = np.abs(np.asarray(got, np.float64) - want).max(), np.sqrt((want ** 2).mean())
    assert rms > 0 and err <= tol * rms, (what, err, rms)


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def _expert_bounds(x, W1, W3, W2, dout, w):
    """How far dW1, dW3, dW2 of one expert may be off, element by element, for given rows.  With g = W1 x, u = W3 x, c = w W2^T dout a row adds
    dh1 x^T, dh3 x^T and dout a^T, dh1 = c u silu'(g), dh3 = c silu(g), a = w u silu(g), and v = 2^-8 is half a step of bf16.  g and u are kept in bf16:
    off by v of themselves (and by the adder).  That moves silu'(g) by v |g| / 2 (|silu''| <= 1/2) and silu(g) by 1.1 v |g| (|silu'| <= 1.1).  dh1, dh3
    and a are rounded to bf16 once more.  Products of these errors are below 2 v of the errors.  A row's error times |x| or |dout|, summed, and the adder's
    on top.  (Relative to the RMS of the whole gradient that is no constant: a fifth of the rows here are the same token, whose errors are the
    same and add up.)"""
    x, W1, W3, W2, dout = (t.double() for t in (x, W1, W3, W2, dout))
    v, n = 2.0 ** -8, x.shape[0]
    adder = lambda a, b: _adder(a.shape[1], a.abs() @ b.abs().T)  # noqa: E731
    g, u, c = x @ W1.T, x @ W3.T, w[:, None] * (dout @ W2)
    eg, eu, ec = v * g.abs() + adder(x, W1), v * u.abs() + adder(x, W3), w[:, None] * adder(dout, W2.T) + 2.0 ** -22 * c.abs()
    sig = torch.sigmoid(g)
    silu, slope = g * sig, sig * (1 + g * (1 - sig))
    e1 = c.abs() * (eu * slope.abs() + u.abs() * (eg / 2 + v * slope.abs())) + ec * (u * slope).abs()
    e3 = c.abs() * (1.1 * eg + v * silu.abs()) + ec * silu.abs()
    ea = w[:, None] * (eu * silu.abs() + u.abs() * (1.1 * eg + v * silu.abs()))
    sums = lambda e, value, other: (1 + 2 * v) * (e.T @ other.abs()) + _adder(n, value.abs().T @ other.abs())  # noqa: E731
    return sums(e1, c * u * slope, x), sums(e3, c * silu, x), sums(ea, w[:, None] * u * silu, dout).T


def test_products_of_a_training_step():
    import helpers
    from oracle import rr_oracle as orc
    s = Step(L=2048)          # some hundred tokens for every expert
    s.forward()
    s.check()
    live = (s.ids.view(-1) >= 0).cpu().numpy()          # (the rows of the others are zeros, here and in the oracle)
    _product(s.logits, s.n1, s.Wg.T, "logits")
    _product(s.y, s.n2, s.Wp.T, "y")
    hidden, W1, W3, W2, Wg = (_bits(t) for t in (s.n1, s.W1, s.W3, s.W2, s.Wg))
    a, tokens = s.logits.cpu().numpy(), np.arange(s.T, dtype=np.int32)
    tab = orc.route(a, s.k, s.C, s.G, 3)
    helpers.assert_tables_equal(s.tab, tab, "tables")
    moe, want = s.moe.cpu().numpy(), orc.forward_tokens(hidden, W1, W3, W2, a, tab, tokens)
    _rms(moe[live], want[live], 2e-2, "moe")
    assert not moe[~live].any()
    _, m, r, _ = ref.norm(s.h1, None, None, True, 1e-5)
    _close(s.m2, m, 2 * U * m.abs() + 70 * U * (s.h1.double() - m[:, None]).square().mean(1).sqrt(), "m2")
    _close(s.r2, r, 40 * U * r, "r2")
    # the way back
    s.backward()
    s.check()
    _product(s.dn2, s.dy, s.Wp, "dn2")
    _product(s.dWp, s.dy.T, s.n2, "dWp")
    dh, dl, dW1, dW3, dW2 = (t.cpu().numpy() for t in s.moe_grads)
    dout = _bits(s.dh1)
    want_dh, want_dl = orc.backward_tokens(hidden, W1, W3, W2, dout, a, tab, tokens)
    _rms(dl[live], want_dl[live], 2e-2, "dlogits")
    dWg, gate_dh = orc.gate_bwd(dl.astype(np.float64), hidden, Wg)
    _rms(s.dWg.cpu().numpy(), dWg, 1e-4, "dWg")
    _rms(dh[live], (want_dh + gate_dh)[live], 2e-2, "dhidden of experts and gate")
    assert not dl[~live].any() and not dh[~live].any()
    for e in range(s.E):
        want = orc.backward_expert(hidden, W1, W3, W2, dout, tab, e)
        at = slice(tab.row_offset[e], tab.row_offset[e + 1])
        rows, w = torch.from_numpy(tab.row_token[at]).long().cuda(), torch.from_numpy(tab.row_weight[at]).double().cuda()
        bounds = _expert_bounds(s.n1[rows], s.W1[e], s.W3[e], s.W2[e], s.dh1[rows], w)
        for got, x, tol, what in zip(s.moe_grads[2:], want, bounds, ("dW1", "dW3", "dW2")):
            _close(got[e], torch.from_numpy(x).cuda(), tol, (what, e))
