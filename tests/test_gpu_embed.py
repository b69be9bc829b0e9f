"""rr_embed_fwd / rr_embed_bwd.  Forward: the product in fp32 and one rounding, bit for bit.  Backward: small integers, whose sums fp32 holds
exactly, bit for bit; normal deviates against 64 bits with half a step of the type and u = 2^-24 of the sum of magnitudes for each step of a sum (32 in
a chunk, 8 rows and n / 256 parts where a run goes over chunks)."""
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
T = {"f": torch.float32, "b": torch.bfloat16}


def _ids(g, n, V, kind):
    if kind == "one":
        return torch.full((n,), V - 1, device="cuda")
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    if kind == "few":      # half of them one id, the rest spread
        ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, torch.full_like(ids, V // 3), ids)
    if kind == "gaps":     # a padded batch
        ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.3, torch.full_like(ids, -1), ids)
    if kind == "none":
        ids = torch.full_like(ids, -1)
    return ids


SIZES = [(1, 1, 1), (1, 7, 8), (5, 3, 1000), (31, 100, 64), (32, 32000, 256), (33, 5, 2056), (37, 9, 4096), (128, 40, 520), (129, 40, 520), (100, 3000, 2064), (1000, 300, 7), (1501, 9973, 1000), (2048, 2, 128), (2049, 65535, 24),
         (4097, 65536, 8), (9000, 70000, 40), (16384, 1 << 17, 16), (16385, 50, 72), (40001, 262144, 9), (65536, 32000, 8)]


@pytest.mark.parametrize("n,V,d", SIZES)
def test_forward(n, V, d):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(n + V + d)
    for i, (tt, yt) in enumerate((("f", "f"), ("f", "b"), ("b", "f"), ("b", "b"))):
        table = torch.randn(V, d, generator=g, device="cuda").to(T[tt])
        ids = _ids(g, n, V, ("gaps", "few", "one", "none")[i])
        ids = ids if i % 2 else ids.int()
        for pad, scale in ((0, 1.0), (8, -0.37), (3, 32.0)):
            whole = torch.full((n + 1, d + pad), 7.0, device="cuda", dtype=T[yt])
            y = rr.embed_fwd(ids, table, scale=scale, out=whole[:n, :d])
            want = torch.where((ids >= 0)[:, None], table.float()[ids.clamp(min=0).long()] * torch.tensor(scale, device="cuda"), torch.zeros((), device="cuda")).to(T[yt])
            assert torch.equal(y, want)
            assert (whole[n:] == 7).all() and (whole[:, d:] == 7).all()
            rr.check(y._workspace)


@pytest.mark.parametrize("kind", ["spread", "few", "one", "gaps", "none"])
@pytest.mark.parametrize("n,V,d", SIZES)
def test_gradient(n, V, d, kind):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(n * 3 + V + d)
    ids = _ids(g, n, V, kind)
    ws = rr.alloc_workspace(rr.embed_workspace_bytes(n, V, d)[1])
    for i, (yt, tt) in enumerate((("f", "f"), ("f", "b"), ("b", "f"), ("b", "b"))):
        pad, scale, add = (0, 8, 3, 0)[i], (1.0, 0.5, 2.0, -1.0)[i], i % 2 == 1
        at = ids if i % 2 else ids.int()
        whole = torch.full((V * d + 8,), 7.0, device="cuda", dtype=T[tt])
        dtable = whole[:V * d].view(V, d)
        old = torch.randint(-4, 5, (V, d), generator=g, device="cuda").to(T[tt])
        if add:
            dtable.copy_(old)
        # integers: exact sums, one rounding
        dy = torch.randint(-3, 4, (n, d + pad), generator=g, device="cuda").to(T[yt])[:, :d]
        dy = torch.where((at >= 0)[:, None], dy, torch.full((), float("nan"), device="cuda", dtype=T[yt]))      # nothing has cleared the padding
        if pad:
            wide = torch.empty(n, d + pad, device="cuda", dtype=T[yt])
            wide[:, :d] = dy
            dy = wide[:, :d]
        rr.embed_bwd(at, dy, dtable, scale=scale, accumulate=add, workspace=ws)
        rr.check(ws)
        want, _ = ref.embed_gradient(at, dy, V, scale)
        assert torch.equal(dtable, (want + old.double() if add else want).to(T[tt])), (yt, tt)
        assert (whole[V * d:] == 7).all()
        # normal deviates
        dy = torch.randn(n, d, generator=g, device="cuda").to(T[yt])
        got = rr.embed_bwd(at, dy, torch.empty(V, d, device="cuda", dtype=T[tt]), scale=scale, workspace=ws)
        want, size = ref.embed_gradient(at, dy, V, scale)
        tol = torch.finfo(T[tt]).eps / 2 * want.abs() + (44 + n / 256) * U * size
        assert ((got.double() - want).abs() <= tol).all(), (yt, tt)
        assert torch.equal(rr.embed_bwd(at, dy, torch.empty_like(got), scale=scale), got)       # the same bits again, from another workspace


def test_ids_outside_the_table():
    import paper_2402_12399_b200 as rr
    V, d = 50, 24
    table = torch.randn(V, d, device="cuda")
    dy = torch.ones(6, d, device="cuda")
    for bad, dtype in ((V, torch.int32), (-2, torch.int32), ((1 << 31) - 1, torch.int32), (-(1 << 31), torch.int32), (V, torch.int64), (1 << 32, torch.int64),
                       ((1 << 32) + 3, torch.int64), (-(1 << 63), torch.int64), ((1 << 63) - 1, torch.int64)):
        ids = torch.tensor([3, bad, 4, -1, 3, 49], dtype=dtype, device="cuda")
        y = rr.embed_fwd(ids, table)
        with pytest.raises(rr.RRError) as e:
            rr.check(y._workspace)
        assert e.value.code == 1
        rr.check(y._workspace)
        assert (y[1] == 0).all() and (y[3] == 0).all() and torch.equal(y[0], table[3]) and torch.equal(y[5], table[49])
        for add in (False, True):
            g = rr.embed_bwd(ids, dy, torch.zeros(V, d, device="cuda"), accumulate=add)
            with pytest.raises(rr.RRError):
                rr.check(g._workspace)
            assert (g[3] == 2).all() and (g[4] == 1).all() and (g[49] == 1).all() and float(g.sum()) == 4 * d


def test_no_tokens():
    import paper_2402_12399_b200 as rr
    table, ids, dy = torch.ones(5, 8, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, 8, device="cuda")
    assert rr.embed_fwd(ids, table).shape == (0, 8)
    assert (rr.embed_bwd(ids, dy, table, accumulate=True) == 1).all()
    assert (rr.embed_bwd(ids, dy, table) == 0).all()


def test_ids_of_any_shape():
    import paper_2402_12399_b200 as rr
    table, ids = torch.randn(10, 16, device="cuda"), torch.randint(0, 10, (3, 4), device="cuda")
    assert torch.equal(rr.embed_fwd(ids, table), table[ids.view(-1)])


def test_tables_beyond_32_bits():
    """a table of 2^32 elements and more: the last rows"""
    import paper_2402_12399_b200 as rr
    V, d = 1100000, 4096
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    table = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    table[-2:].normal_()
    ids = torch.tensor([V - 1, 0, V - 2, V - 1, -1], device="cuda")
    y = rr.embed_fwd(ids, table)
    assert torch.equal(y[0], table[-1]) and torch.equal(y[2], table[-2]) and (y[1] == 0).all() and (y[4] == 0).all()
    table.fill_(3)
    dy = torch.randint(-3, 4, (5, d), device="cuda").bfloat16()
    rr.embed_bwd(ids, dy, table)
    assert torch.equal(table[-1], dy[0] + dy[3]) and torch.equal(table[-2], dy[2]) and torch.equal(table[0], dy[1])
    assert not table[1:1000].any() and not table[-70000:-2].any()


def test_many_tokens():
    """more than 2^20 tokens: many sorted slabs are merged; exact on integers"""
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(9)
    n, V, d = (1 << 20) + 77, 5003, 8
    ids = _ids(g, n, V, "few")
    dy = torch.randint(-3, 4, (n, d), generator=g, device="cuda").bfloat16()
    got = rr.embed_bwd(ids, dy, torch.empty(V, d, device="cuda"))
    assert torch.equal(got, ref.embed_gradient(ids, dy, V, 1.0)[0].float())


def test_captured_with_new_ids():
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(5)
    n, V, d = 3000, 700, 264
    table, ids, dy = torch.randn(V, d, generator=g, device="cuda").bfloat16(), _ids(g, n, V, "few"), torch.randn(n, d, generator=g, device="cuda").bfloat16()
    y, dt = torch.empty(n, d, device="cuda"), torch.empty(V, d, device="cuda")
    a, b = rr.embed_workspace_bytes(n, V, d)
    wa, wb = rr.alloc_workspace(a), rr.alloc_workspace(b)

    def step():
        rr.embed_fwd(ids, table, out=y, workspace=wa)
        rr.embed_bwd(ids, dy, dt, workspace=wb)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for kind in ("gaps", "one", "spread"):
        ids.copy_(_ids(g, n, V, kind))
        dt.fill_(7)
        graph.replay()
        got = y.clone(), dt.clone()
        step()
        assert torch.equal(y, got[0]) and torch.equal(dt, got[1])
        want, size = ref.embed_gradient(ids, dy, V, 1.0)
        assert ((dt.double() - want).abs() <= 60 * U * size).all()


def test_the_binding_refuses():
    import paper_2402_12399_b200 as rr
    t, ids = torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    dy = torch.zeros(4, 8, device="cuda")
    for bad in (lambda: rr.embed_fwd(ids.float(), t), lambda: rr.embed_fwd(ids.cpu(), t), lambda: rr.embed_fwd(ids, t.half()), lambda: rr.embed_fwd(ids, t.t()),
                lambda: rr.embed_fwd(ids, t, out=dy[:3]), lambda: rr.embed_fwd(ids, t, scale=float("inf")), lambda: rr.embed_fwd(ids, t, out=t[:4]),
                lambda: rr.embed_fwd(torch.zeros(8, dtype=torch.int64, device="cuda")[::2], t), lambda: rr.embed_bwd(ids, dy[:3], t), lambda: rr.embed_bwd(ids, dy, t[:, :4]),
                lambda: rr.embed_bwd(ids, t[:4], t), lambda: rr.embed_bwd(ids, dy, t, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((TypeError, ValueError, rr.RRError)):
            bad()
