"""rr_dropout_fwd / rr_dropout_bwd against the published generator and 64-bit arithmetic.

The kernel computes fma(x, factor, residual) in fp32 and rounds once to the result's type: with the factor itself rounded
to fp32, |error| <= eps(type)/2 |y| + 2^-24 |x| factor + 2^-24 |y|, counted below as half a step of the type plus four
half steps of fp32 of the terms."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rng(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def _check(y, x, res, p, rng):
    v = ref.dropped(x.double(), p, rng)
    want = v + (0 if res is None else res.double())
    tol = torch.finfo(y.dtype).eps / 2 * want.abs() + 4 * 2.0 ** -24 * (v.abs() + want.abs())
    bad = (y.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), bad.flatten().nonzero()[:4].tolist())


@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 100003])
@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("yt", ["f32", "bf16"])
def test_forward_and_backward(n, xt, yt):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(n)
    x = torch.randn(n, generator=g, device="cuda").to(TYPES[xt])
    res = torch.randn(n, generator=g, device="cuda").to(TYPES[yt])
    for p in (0.0, 0.1, 0.5, 1.0):
        rng = _rng(n * 77 + 1, -3)                       # the offset's high word is all ones
        guard = torch.full((n + 16,), 7.0, device="cuda", dtype=TYPES[yt])
        out = guard[:n]
        y = rr.dropout_fwd(x, p, rng, residual=res, out=out)
        assert y is out and torch.all(guard[n:] == 7.0)  # nothing behind the end is written
        _check(y, x, res, p, rng)
        _check(rr.dropout_fwd(x, p, rng, out_dtype=TYPES[yt]), x, None, p, rng)
        dx = rr.dropout_bwd(x, p, rng, out_dtype=TYPES[yt])
        _check(dx, x, None, p, rng)
        acc = res.clone()
        rr.dropout_bwd(x, p, rng, out=acc, accumulate=True)
        _check(acc, x, res, p, rng)


def test_in_place_and_no_generator():
    import paper_2402_12399_b200 as rr
    x = torch.randn(5, 1023, device="cuda")
    r = torch.randn(5, 1023, device="cuda").bfloat16()
    rng = _rng(1, 2)
    want = rr.dropout_fwd(x, 0.3, rng, residual=r)
    r2 = r.clone()
    assert torch.equal(rr.dropout_fwd(x, 0.3, rng, residual=r2, out=r2), want)
    x2 = x.clone()
    assert torch.equal(rr.dropout_fwd(x2, 0.3, rng, out=x2), rr.dropout_fwd(x, 0.3, rng))
    assert torch.equal(rr.dropout_fwd(x, 0.0, None), x)
    assert rr.dropout_fwd(x[:0], 0.5, rng).shape == (0, 1023)


def test_nothing_of_a_dropped_element_is_seen():
    import paper_2402_12399_b200 as rr
    rng = _rng(11, 0)
    keep = torch.from_numpy(ref.keep_mask(11, 0, 0, 4099, 0.5)[0]).cuda()
    x = torch.where(keep, torch.ones(4099, device="cuda"), torch.tensor(float("nan"), device="cuda"))
    y = rr.dropout_fwd(x, 0.5, rng)
    assert torch.equal(y, torch.where(keep, 2.0, 0.0))
    x[~keep] = float("-inf")
    assert torch.equal(rr.dropout_bwd(x, 0.5, rng), y)


def test_index_beyond_32_bits_of_bytes():
    """n > 2^32: the counter's high part and 64-bit addresses; only the two ends are compared."""
    import paper_2402_12399_b200 as rr
    n = (1 << 32) + 12345
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    rng = _rng(123456789123, 5)
    y = rr.dropout_fwd(x, 0.5, rng)
    for first in (0, (1 << 32) - 1000, n - 5000):
        m = min(5000, n - first)
        want = ref.keep_mask(123456789123, 5, first, m, 0.5)[0]
        assert torch.equal(y[first:first + m].cpu(), torch.from_numpy(want).to(torch.bfloat16) * 2)


def test_captured_call_reads_the_generator_at_replay():
    import paper_2402_12399_b200 as rr
    x = torch.randn(3000, device="cuda")
    rng, out = _rng(5, 0), torch.empty(3000, device="cuda")
    rr.dropout_fwd(x, 0.5, rng, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rr.dropout_fwd(x, 0.5, rng, out=out)
        rng[1:].add_(1)
    seen = []
    for _ in range(3):
        want = ref.dropped(x.double(), 0.5, rng)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.double(), want.float().double())
        seen.append(out.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_another_stream():
    import paper_2402_12399_b200 as rr
    x, rng = torch.randn(1 << 20, device="cuda"), _rng(3, 4)
    want = rr.dropout_fwd(x, 0.2, rng)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = rr.dropout_fwd(x, 0.2, rng)
    side.synchronize()
    assert torch.equal(got, want)


def test_binding_refuses():
    import paper_2402_12399_b200 as rr
    x, rng = torch.randn(8, 8, device="cuda"), _rng(1, 1)
    for call, err in [(lambda: rr.dropout_fwd(x, 0.5, None), ValueError), (lambda: rr.dropout_fwd(x, 1.5, rng), rr.RRError),
                      (lambda: rr.dropout_fwd(x, float("nan"), rng), rr.RRError), (lambda: rr.dropout_fwd(x, -0.1, rng), rr.RRError),
                      (lambda: rr.dropout_fwd(x.half(), 0.5, rng), TypeError), (lambda: rr.dropout_fwd(x.T[:4], 0.5, rng), ValueError),
                      (lambda: rr.dropout_fwd(x, 0.5, rng.int()), TypeError), (lambda: rr.dropout_fwd(x, 0.5, rng, residual=x[:4]), ValueError),
                      (lambda: rr.dropout_fwd(x, 0.5, rng, residual=x.bfloat16(), out=torch.empty_like(x)), TypeError),
                      (lambda: rr.dropout_fwd(x.cpu(), 0.5, rng), ValueError), (lambda: rr.dropout_bwd(x, 0.5, rng, accumulate=True), ValueError),
                      (lambda: rr.dropout_fwd(x.view(-1)[1:], 0.5, rng), rr.RRError)]:
        with pytest.raises(err):
            call()
