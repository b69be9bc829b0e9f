"""Gradients of parameters that lie back to back in one buffer, whatever their sizes: the clip takes such a list, and the norm's and the embedding's
gradients are written into it, the same bits as into buffers of their own."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu
T = {"f": torch.float32, "b": torch.bfloat16}


def _flat(n, at, dtype=torch.float32):
    """n elements from element `at` of a buffer of sevens on"""
    whole = torch.full((at + n + 9,), 7.0, device="cuda", dtype=dtype)
    return whole, whole[at:at + n]


@pytest.mark.parametrize("M,N", [(1, 1), (1, 4096), (3, 2056), (2, 9000), (1, 20000), (4, 64), (300, 40), (700, 1024), (33, 1023), (700, 5000)])
def test_norm(M, N):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(M + N)
    for (yt, ht), at, add, both in itertools.product(("bb", "fb"), (1, 2, 3), (False, True), (True, False)):
        dy, h, w = (torch.randn(*s, generator=g, device="cuda").to(T[t]) for s, t in (((M, N), yt), ((M, N), ht), ((N,), "b")))
        mean, rstd = h.float().mean(1), 1 / (h.float().var(1, unbiased=False) + 1e-5).sqrt()
        old = torch.randn(2, N, generator=g, device="cuda")
        want = rr.norm_bwd(dy, h, w, mean, rstd, dw=old[0].clone(), dbias=old[1].clone(), dx=torch.empty_like(h), add_dw=add)
        (ww, dw), (wb, db) = _flat(N, at), _flat(N, 4 - at)
        dw.copy_(old[0])
        db.copy_(old[1])
        dx = torch.empty_like(h)
        rr.norm_bwd(dy, h, w, mean, rstd, dw=dw, dbias=db if both else None, dx=dx, add_dw=add)
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2] if both else old[1])
        for whole, first in ((ww, at), (wb, 4 - at)):
            assert (whole[:first] == 7).all() and (whole[first + N:] == 7).all()


@pytest.mark.parametrize("n,V,d", [(1, 3, 1), (5, 9, 1000), (128, 40, 520), (129, 40, 520), (1501, 9973, 100), (20000, 50, 72), (300, 700, 8)])
@pytest.mark.parametrize("yt", "fb")
@pytest.mark.parametrize("tt", "fb")
def test_embedding(n, V, d, yt, tt):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(n + V)
    ids = torch.randint(-1, V, (n,), generator=g, device="cuda")
    ids[n // 2:] = V // 2
    # small integers: exact sums, whatever their order (2 x 3 x 20000 stays below 2^24)
    dy = torch.randint(-3, 4, (n, d), generator=g, device="cuda").to(T[yt])
    for at, add in itertools.product((1, 2, 5, 7), (False, True)):
        old = torch.randint(-4, 5, (V, d), generator=g, device="cuda").to(T[tt])
        want = rr.embed_bwd(ids, dy, old.clone(), scale=2.0, accumulate=add)
        whole, flat = _flat(V * d, at, T[tt])
        flat.copy_(old.view(-1))
        got = rr.embed_bwd(ids, dy, flat.view(V, d), scale=2.0, accumulate=add)
        rr.check(got._workspace)
        assert torch.equal(got, want)
        assert (whole[:at] == 7).all() and (whole[at + V * d:] == 7).all()
    flat.fill_(3)
    assert (rr.embed_bwd(ids[:0], dy[:0], flat.view(V, d)) == 0).all() and (whole[:at] == 7).all() and (whole[at + V * d:] == 7).all()


def test_one_buffer_for_a_step():
    """Table, weight and bias back to back with odd sizes: gradients into it, then the clip of the same views."""
    import paper_2402_12399_b200 as rr
    n, V, d = 700, 101, 37
    g = torch.Generator("cuda").manual_seed(1)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    x, dy, w = torch.randn(n, d, generator=g, device="cuda"), torch.randn(n, d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    flat = torch.full((1 + V * d + 2 * d + 1,), 7.0, device="cuda")
    table, dw, db = flat[1:1 + V * d].view(V, d), flat[1 + V * d:1 + V * d + d], flat[1 + V * d + d:-1]
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    rr.norm_fwd(x, w, mean=mean, rstd=rstd)
    dx = rr.norm_bwd(dy, x, w, mean, rstd, dx=torch.empty_like(x), dw=dw, dbias=db)[0]
    rr.embed_bwd(ids, dx, table)
    own = rr.norm_bwd(dy, x, w, mean, rstd, dw=torch.empty(d, device="cuda"), dbias=torch.empty(d, device="cuda"))[1:]
    apart = rr.embed_bwd(ids, dx, torch.empty(V, d, device="cuda"))
    assert torch.equal(table, apart) and torch.equal(dw, own[0]) and torch.equal(db, own[1])
    norm = rr.clip_grads([table, dw, db], 0.5)
    want = torch.cat([apart.view(-1), *own]).double()
    size = want.norm()
    # (the norm to 4 u and its rounding, the factor as much, a product's rounding)
    assert abs(float(norm[0]) - size) <= 6 * 2.0 ** -24 * size
    want *= 0.5 / (size + 1e-6)
    assert ((flat[1:-1].double() - want).abs() <= 8 * 2.0 ** -24 * want.abs()).all() and flat[0] == 7 and flat[-1] == 7

