"""rr_grad_plan / rr_clip_grads against 64-bit arithmetic.  u = 2^-24: eight squares are added in fp32 (8 u of their sum), the rest in 64 bits, so
the norm is off by 4 u and its rounding, the factor by as much; a gradient by half a step of its type and 8 u."""
import math

import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
T = {"f": torch.float32, "b": torch.bfloat16}


def _check(out, grads, norm, bound):
    n, f = ref.clip(grads, bound)
    assert abs(float(norm[0]) - n) <= 6 * U * n and abs(float(norm[1]) - f) <= 6 * U * f, (norm.tolist(), n, f)
    for o, g in zip(out, grads):
        if o is None:
            continue
        want = g.double() * f
        tol = torch.finfo(o.dtype).eps / 2 * want.abs() + 8 * U * want.abs() + 1e-44
        assert ((o.double() - want).abs() <= tol).all()


LISTS = [[1], [7, 1, 8], [2048], [2049, 0, 3], [8192, 100000], [5, 65536, 12, 0, 0, 77777, 1], [3] * 300, [1000003, 17, 4096 * 512], [0, 0], [], [1 << 23]]


@pytest.mark.parametrize("sizes", LISTS, ids=[f"{len(s)}x{max(s, default=0)}" for s in LISTS])
@pytest.mark.parametrize("st", "fb")
@pytest.mark.parametrize("dt", ["same", "f", "b"])
def test_clip(sizes, st, dt):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(len(sizes) + sum(sizes))
    for flat in (0, 1, 3):     # each by itself; back to back, from an odd element on
        if flat:
            whole = torch.full((sum(sizes) + flat + 9,), 7.0, device="cuda", dtype=T[st])
            at, grads = flat, []
            for n in sizes:
                grads.append(whole[at:at + n])
                grads[-1].copy_(torch.randn(n, generator=g, device="cuda"))
                at += n
        else:
            grads = [torch.randn(n, generator=g, device="cuda").to(T[st]) for n in sizes]
        before = [t.clone() for t in grads]
        total, _ = ref.clip(before, 1.0)
        out = None if dt == "same" else [torch.full((n,), 7.0, device="cuda", dtype=T[dt]) for n in sizes]
        plan = rr.grad_plan(grads, out=out)
        norm = rr.clip_grads(plan, float("inf"))
        rr.check(norm._workspace)
        _check(plan.out, before, norm, math.inf)
        assert norm[1] == 1 and (dt != "same" or all(torch.equal(a, b) for a, b in zip(grads, before)))
        norm = rr.clip_grads(plan, total / 3 + 1e-3)
        _check(plan.out, before, norm, total / 3 + 1e-3)
        if flat:
            assert (whole[:flat] == 7).all() and (whole[at:] == 7).all()
        if dt != "same":
            again = [t.clone() for t in plan.out]
            for t in plan.out:
                t.fill_(7)
            second = rr.clip_grads(plan, total / 3 + 1e-3)
            assert torch.equal(second, norm) and all(torch.equal(a, b) for a, b in zip(again, plan.out))


def test_mixed_types_and_tensors_that_only_count():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(1)
    grads = [torch.randn(n, generator=g, device="cuda").to(T["fb"[i % 2]]) for i, n in enumerate((1001, 64, 30000, 5, 8191))]
    keep = [t.clone() for t in grads]
    out = [torch.empty(1001, device="cuda", dtype=torch.bfloat16), None, grads[2], torch.empty(5, device="cuda"), None]
    plan = rr.grad_plan(grads, out=out)
    _check(plan.out, keep, rr.clip_grads(plan, 2.0), 2.0)
    assert torch.equal(grads[1], keep[1]) and torch.equal(grads[4], keep[4])


def test_a_plain_list_is_clipped_in_place():
    import paper_2402_12399_b200 as rr
    grads = [torch.randn(100, 7, device="cuda"), torch.randn(64, device="cuda").bfloat16()]
    keep = [t.clone() for t in grads]
    _check(grads, keep, rr.clip_grads(grads, 1.0), 1.0)


@pytest.mark.parametrize("types", ["ff", "bb", "fb", "bf"])
@pytest.mark.parametrize("n", [1, 9, 2047, 2048 + 8, 3 * 8192 + 5, 1 << 23])
def test_buffers_without_a_common_boundary(types, n):
    """src begins one to seven elements behind a 16-byte boundary and dst at one, and the other way round."""
    import paper_2402_12399_b200 as rr
    for s, d in ((1, 0), (0, 1), (3, 2), (7, 0), (0, 7)):
        g = torch.Generator("cuda").manual_seed(n + s)
        src = torch.randn(n + s, generator=g, device="cuda").to(T[types[0]])[s:]
        whole = torch.full((n + d + 9,), 7.0, device="cuda", dtype=T[types[1]])
        keep, out = src.clone(), whole[d:d + n]
        plan = rr.grad_plan([src], out=[out])
        norm = rr.clip_grads(plan, 0.5)
        rr.check(norm._workspace)
        _check([out], [keep], norm, 0.5)
        assert torch.equal(src, keep) and (whole[:d] == 7).all() and (whole[d + n:] == 7).all()


@pytest.mark.parametrize("t", "fb")
@pytest.mark.parametrize("size", [1e30, 3e38, 1e-30, 1e-40, 0.0])
def test_squares_that_fp32_cannot_hold(t, size):
    import paper_2402_12399_b200 as rr
    for n in (1, 9, 50021):
        x = (torch.rand(n, device="cuda") * 0.5 + 0.5).mul_(size).to(T[t])
        y = torch.empty(n, device="cuda")
        norm = rr.clip_grads(rr.grad_plan([x], out=[y]), size)
        rr.check(norm._workspace)
        want, f = ref.clip([x], size)
        assert float(norm[0]) == pytest.approx(want, rel=6 * U, abs=1e-45) if want < 3.4e38 else float(norm[0]) == math.inf
        assert float(norm[1]) == pytest.approx(f, rel=6 * U, abs=1e-45)
        assert torch.isfinite(y).all()
    # among ordinary ones: nothing of the small is lost to the large, nothing overflows
    x = torch.cat([torch.full((16,), 1e-25, device="cuda"), torch.full((16,), 1e25, device="cuda")]).to(T[t])
    norm = rr.clip_grads([x], math.inf)
    assert float(norm[0]) == pytest.approx(ref.clip([x], 1.0)[0], rel=6 * U)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_gradients_that_are_not_finite(bad):
    import paper_2402_12399_b200 as rr
    for n, at in ((1, 0), (9, 8), (100001, 100000), (100001, 4096)):
        x = torch.randn(n, device="cuda")
        x[at] = bad
        keep, y = x.clone(), torch.empty(n, device="cuda")
        for plan in (rr.grad_plan([torch.ones(5, device="cuda"), x]), rr.grad_plan([x], out=[y])):
            norm = rr.clip_grads(plan, 1e-3)
            with pytest.raises(rr.RRError) as e:
                rr.check(norm._workspace)
            assert e.value.code == 5
            assert not math.isfinite(float(norm[0])) and float(norm[1]) == 1
            same = plan.out[-1].view(torch.int32) == keep.view(torch.int32)
            if plan.out[-1] is y:     # (a copy's NaN has gone through a product, which gives it another payload)
                same |= torch.isnan(y) & torch.isnan(keep)
            assert same.all()


def test_bounds():
    import paper_2402_12399_b200 as rr
    x = torch.full((100,), 0.5, device="cuda")
    assert float(rr.clip_grads([x], 5.0)[1]) < 1                       # norm 5: the 1e-6 in the factor
    assert float(rr.clip_grads([x.fill_(0.5)], 5.1)[1]) == 1 and (x == 0.5).all()
    assert float(rr.clip_grads([x], 0.0)[1]) == 0 and not x.any()
    assert rr.clip_grads([x], 1.0).tolist() == [0, 1]


def test_more_elements_than_32_bits_count():
    import paper_2402_12399_b200 as rr
    n = (1 << 32) + 4099
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    norm = rr.clip_grads([x], float(n) ** 0.5 / 4)
    assert float(norm[0]) == pytest.approx(n ** 0.5, rel=6 * U)
    assert (x[-5000:] == 0.25).all() and (x[:5000] == 0.25).all() and (x[(1 << 32) - 100:(1 << 32) + 100] == 0.25).all()


def test_more_tensors_than_are_looked_up_at_once():
    import paper_2402_12399_b200 as rr
    for count, size in ((70000, 3), (700, 5000)):
        whole = torch.randn(count * size + 1, device="cuda")[1:]
        keep = whole.clone()
        grads = list(whole.view(count, size).unbind(0))
        _check([whole], [keep], rr.clip_grads(rr.grad_plan(grads), 7.0), 7.0)


def test_plans_one_after_the_other_at_one_address():
    """A plan that takes the place of the last one at once: nothing of the old list is seen."""
    import paper_2402_12399_b200 as rr
    grads = [[torch.randn(257 * (i + 1) + 31 * j, device="cuda") for j in range(1 + i % 7)] for i in range(30)]
    keep = [[t.clone() for t in g] for g in grads]
    norms = torch.empty(30, 2, device="cuda")
    ws = rr.alloc_workspace(rr.clip_workspace_bytes())
    torch.cuda.synchronize()
    for i, g in enumerate(grads):
        norms[i] = rr.clip_grads(rr.grad_plan(g), 1.0, workspace=ws)     # (the plan's buffer goes back to the allocator, which hands it out again)
    for i, g in enumerate(grads):
        _check(g, keep[i], norms[i], 1.0)


def test_captured_with_new_gradients():
    import paper_2402_12399_b200 as rr
    grads = [torch.randn(3000, device="cuda"), torch.randn(77, 9, device="cuda").bfloat16()]
    norm, ws = torch.empty(2, device="cuda"), rr.alloc_workspace(rr.clip_workspace_bytes())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan = rr.grad_plan(grads)          # (made inside: kernels, no copy from host memory)
        rr.clip_grads(plan, 1.0, norm=norm, workspace=ws)
    for s in (0.001, 1.0, 50.0):
        for t in grads:
            t.copy_(s * torch.randn(t.shape, device="cuda"))
        keep = [t.clone() for t in grads]
        graph.replay()
        _check(grads, keep, norm, 1.0)


def test_the_binding_refuses():
    import paper_2402_12399_b200 as rr
    x = torch.zeros(64, device="cuda")
    p = rr.grad_plan([x])
    for bad in (lambda: rr.grad_plan([x, x]), lambda: rr.grad_plan([x[:32], x[31:]]), lambda: rr.grad_plan([x[::2]]), lambda: rr.grad_plan([x.half()]),
                lambda: rr.grad_plan([x], out=[x[:63]]), lambda: rr.grad_plan([x[:32]], out=[x[16:48]]), lambda: rr.grad_plan([x.cpu()]),
                lambda: rr.grad_plan([x[:16], x[16:32]], out=[x[32:48], x[40:56]]), lambda: rr.clip_grads(p, -1.0), lambda: rr.clip_grads(p, float("nan")),
                lambda: rr.clip_grads(p, 1.0, norm=x), lambda: rr.clip_grads(p, 1.0, norm=torch.zeros(2, dtype=torch.float64, device="cuda")),
                lambda: rr.clip_grads(p, 1.0, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((TypeError, ValueError, rr.RRError)):
            bad()
