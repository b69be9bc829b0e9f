"""The embedding and its gradient where blocks go round their loops several times: units and pieces of rows beyond 16 tiles an SM, zeroed rows beyond
one bitmap, long runs beyond four blocks an SM.  Products and sums of small whole numbers are exact, so all is equal bit for bit."""
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
T = {"f": torch.float32, "b": torch.bfloat16}


# narrow rows (units; more than 2368 tiles of 1024 of them): a row of one, three, five, nine units; wide ones (more than 18944 pieces): one, two, three, five to a row
@pytest.mark.parametrize("tt", "fb")
@pytest.mark.parametrize("yt", "fb")
@pytest.mark.parametrize("n,d", [(2500003, 8), (900001, 12), (600001, 40), (300001, 9), (20011, 1024), (10007, 2048), (7001, 2816), (4003, 5000), (20011, 512), (20011, 127)])
def test_forward(n, d, tt, yt):
    import paper_2402_12399_b200 as rr
    g = torch.Generator("cuda").manual_seed(n)
    V = 3001
    table = torch.randint(-100, 101, (V, d), generator=g, device="cuda").to(T[tt])
    ids = torch.randint(-1, V, (n,), generator=g, device="cuda")
    for pad in (0, 8, 3):
        whole = torch.full((n + 1, d + pad), 7.0, device="cuda", dtype=T[yt])
        y = rr.embed_fwd(ids if pad else ids.int(), table, scale=0.5, out=whole[:n, :d])
        rr.check(y._workspace)
        want = torch.where((ids >= 0)[:, None], table.float()[ids.clamp(min=0)] * 0.5, torch.zeros((), device="cuda")).to(T[yt])
        assert torch.equal(y, want), pad
        assert (whole[n:] == 7).all() and (whole[:, d:] == 7).all()


def _check_gradient(n, V, d, yt, tt, ids, g):
    import paper_2402_12399_b200 as rr
    dy = torch.randint(-2, 3, (n, d), generator=g, device="cuda").to(T[yt])
    got = rr.embed_bwd(ids, dy, torch.full((V, d), 7.0, device="cuda", dtype=T[tt]))
    rr.check(got._workspace)
    assert torch.equal(got, ref.embed_gradient(ids, dy, V, 1.0)[0].to(T[tt]))


@pytest.mark.parametrize("V,d", [(1 << 26, 1), ((1 << 26) - 3, 1), (50000001, 2)])
@pytest.mark.parametrize("n", [100, 5000])
def test_rows_to_zero_beyond_one_bitmap(n, V, d):
    """(592 blocks beside 100 tokens, 147 beside a sort: up to 457000 rows each, and 2^18 in a bitmap; 592 have fewer)"""
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    g = torch.Generator("cuda").manual_seed(n)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    ids[:4] = torch.tensor([0, V - 1, 1 << 18, (1 << 18) - 1])
    _check_gradient(n, V, d, "b", "b", ids, g)


@pytest.mark.parametrize("yt,tt", ["ff", "bf", "bb", "fb"])
@pytest.mark.parametrize("n,V,d", [(30000, 50, 4100), (30000, 50, 4104), (30000, 60, 2700), (9000, 100, 2049)])
def test_long_runs(n, V, d, yt, tt):
    """50 and more ids with 90 to 600 tokens each, in 9 to 17 tiles of columns: more items than the 592 blocks that join pieces"""
    g = torch.Generator("cuda").manual_seed(V + d)
    _check_gradient(n, V, d, yt, tt, torch.randint(0, V, (n,), generator=g, device="cuda"), g)


@pytest.mark.parametrize("d", [8, 300, 1030, 2050])
def test_runs_of_every_length(d):
    """Runs of 1 to 200 tokens, one after the other in the sorted order, so that they begin everywhere in their chunks (8, 16 and 32 tokens long) and
    end everywhere around the length from which they are cut into pieces."""
    g = torch.Generator("cuda").manual_seed(d)
    for copies in (1, 4):
        length = torch.cat([torch.arange(1, 201) for _ in range(copies)])
        ids = torch.repeat_interleave(torch.arange(len(length)), length)
        ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(1))].cuda()
        _check_gradient(len(ids), len(length) + 3, d, "b", "f", ids, g)
