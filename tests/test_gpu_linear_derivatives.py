"""rr_linear_bwd against derivatives of the forward definition in 64 bits, mask, bias and saved pre-activations included.

The wanted gradients come from the definition of y alone: central differences (every element of a small layer) and autograd in 64
bits (whose agreement with the differences is tested on the CPU).  No slope formula and no z of the kernel enters them.  Bound per element, with
f the factor of kept elements, HALF = 2^-8 half a step of bf16 and C >= |act''|:
  - z is saved in bf16 and summed by the tensor cores' adder: its error e_z = HALF |z| + (K/16 + 8) 2^-23 sum |x w|, and dz moves by
    f |dy| C e_z; the slope's own arithmetic adds f |dy| 4e-6 (1 + |z|);
  - dz is rounded to bf16 (not without an activation): HALF of itself;
  - these errors pass through the product with their signs unknown: sum over the contraction of error x |other factor|;
  - the adder again, (n/16 + 8) 2^-23 of the sum of magnitudes, and 2^-22 of the value for the fp32 result.
C: ReLU 0 (rounding to bf16 crosses no zero; where |z| lies within the adder's error the slope may be 0 or 1), GELU 2 phi(0) = 0.798 at v = 0 and its tanh form within 1 %
of that (0.81), SiLU 1/2 at v = 0."""
import pytest
import torch

import block_ref as ref

CURVE = (0.0, 0.0, 0.798, 0.81, 0.5)
HALF = 2.0 ** -8
P = 0.25


def _layer(M, N, K, seed):
    g = torch.Generator().manual_seed(seed)
    x, w = torch.randn(M, K, generator=g).bfloat16(), (torch.randn(N, K, generator=g) * 2 * K ** -0.5).bfloat16()
    b, dy = torch.randn(N, generator=g).bfloat16(), torch.randn(M, N, generator=g).bfloat16()
    keep = ref.dropped(torch.ones(M, N, dtype=torch.float64), P, torch.tensor([seed, 7]))     # 0 or the factor
    return x, w, b, dy, keep


def _wanted(x, w, b, dy, keep, act):
    at = [t.double().requires_grad_() for t in (x, w, b)]
    y = ref.act(at[0] @ at[1].T + at[2], act) * keep
    (y * dy.double()).sum().backward()
    return [t.grad for t in at]


def _bounds(x, w, b, dy, keep, act):
    x, w, b, dy = (t.double() for t in (x, w, b, dy))
    (M, K), N = x.shape, w.shape[0]
    z = x @ w.T + b
    adder = (K / 16 + 8) * 2.0 ** -23 * (x.abs() @ w.abs().T + b.abs())
    e_z = HALF * z.abs() + adder
    dz = dy.abs() * keep * (1.13 if act else 1.0)                              # |act'| <= 1.13
    moved = dy.abs() * keep * (CURVE[act] * e_z + 4e-6 * (1 + z.abs())) if act else torch.zeros_like(z)
    if act == 1:
        moved = torch.where(z.abs() <= adder, dy.abs() * keep, moved)
    rounded = moved + HALF * (dz + moved) if act else moved

    def product(err, mag, other, n):
        return err @ other + ((n / 16 + 8) * 2.0 ** -23 + 2.0 ** -22) * (mag @ other)
    return (product(rounded, dz, w.abs(), N), product(rounded.T, dz.T, x.abs(), M), moved.sum(0) + (M / 8 + 16) * 2.0 ** -24 * dz.sum(0))


def _right(got, want, bound):
    """share of the elements within their bounds"""
    return float(((got.double().cpu() - want).abs() <= bound).double().mean())


@pytest.mark.parametrize("act", range(5))
def test_autograd_agrees_with_differences_and_the_bounds_refuse_wrong_gradients(act):
    x, w, b, dy, keep = _layer(9, 24, 16, 2)
    want, bounds = _wanted(x, w, b, dy, keep, act), _bounds(x, w, b, dy, keep, act)
    at = [t.double() for t in (x, w, b)]

    def loss(t):
        return float((dy.double() * keep * ref.act(t[0] @ t[1].T + t[2], act)).sum())
    h = 1e-6
    for i, t in enumerate(at):
        flat = t.view(-1)
        diff = torch.empty_like(flat)
        for j in range(flat.numel()):
            kept = float(flat[j])
            flat[j] = kept + h
            up = loss(at)
            flat[j] = kept - h
            diff[j] = (up - loss(at)) / (2 * h)
            flat[j] = kept
        # (the loss is some 100 in magnitude: its rounding, 1e-14, over 2e-6, and the third derivative's h^2)
        assert torch.allclose(diff.view_as(t), want[i], rtol=1e-6, atol=1e-6)
    for g, bound in zip(want, bounds):
        assert _right(g, g, bound) == 1
        for wrong in (torch.zeros_like(g), -g, 2 * g, g * 0.75, g.roll(1, -1)):
            assert _right(wrong, g, bound) < 0.6, act


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(9, 24, 16), (300, 136, 72), (1, 64, 264), (130, 24, 520)])
@pytest.mark.parametrize("act", range(5))
def test_every_gradient(M, N, K, act):
    import paper_2402_12399_b200 as rr
    x, w, b, dy, keep = _layer(M, N, K, 2)
    want, bounds = _wanted(x, w, b, dy, keep, act), _bounds(x, w, b, dy, keep, act)
    gx, gw, gb, gdy = (t.cuda() for t in (x, w, b, dy))
    rng = torch.tensor([2, 7], device="cuda")
    z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    rr.linear_fwd(gx, gw, gb, act=act, p=P, rng=rng, z=z)
    got = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    rr.linear_bwd(gdy, gx, gw, z, act=act, p=P, rng=rng, dx=got[0], dw=got[1], dbias=got[2])
    for name, g, v, bound in zip(("dx", "dw", "dbias"), got, want, bounds):
        assert _right(g, v, bound) == 1, (name, float(((g.double().cpu() - v).abs() / bound.clamp(min=1e-30)).max()))
