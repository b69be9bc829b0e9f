"""What the C entry points of the operators around the expert layer refuse, before any pointer is touched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def rr():
    from paper_2402_12399_b200 import binding, build
    build.build()
    binding.lib()
    return binding


AT, ODD = 4096, 4096 + 8       # never dereferenced: a 256-byte aligned address and one that is not even 16-byte aligned


def _linear(rr, **kw):
    s = dict(M=16, N=24, K=64, act=0, y_dtype=0, dx_dtype=0, dw_dtype=0, flags=0, p=0.0, ldx=0, ldr=0, ldy=0, ldz=0, lddy=0, lddx=0)
    s.update({k: v for k, v in kw.items() if k in s})
    return rr._CLinear(*s.values())


def test_dropout(rr):
    f, b = rr.lib().rr_dropout_fwd, rr.lib().rr_dropout_bwd
    ok = dict(n=8, xt=0, yt=1, x=AT, r=None, p=0.5, rng=AT, y=2 * AT)
    for bad in [dict(n=-1), dict(xt=2), dict(yt=-1), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(rng=None), dict(rng=ODD), dict(x=None),
                dict(y=None), dict(x=ODD), dict(y=ODD), dict(r=ODD), dict(x=2 * AT)]:
        a = {**ok, **bad}
        assert f(a["n"], a["xt"], a["yt"], a["x"], a["r"], a["p"], a["rng"], a["y"], None) == 1, bad
        if "r" not in bad:
            assert b(a["n"], a["xt"], a["yt"], a["x"], a["p"], a["rng"], 0, a["y"], None) == 1, bad
    assert f(0, 0, 0, None, None, 0.5, AT, None, None) == 0 and b(0, 0, 0, None, 0.0, None, 1, None, None) == 0


def test_linear_forward(rr):
    f = rr.lib().rr_linear_fwd
    ok = dict(x=AT, w=AT, b=None, r=None, rng=None, y=2 * AT, z=None, ws=AT, n=1 << 20)

    def call(**kw):
        a = {**ok, **kw}
        return f(C.byref(_linear(rr, **kw)), a["x"], a["w"], a["b"], a["r"], a["rng"], a["y"], a["z"], a["ws"], a["n"], None)
    for bad in [dict(M=-1), dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 8), dict(K=(1 << 30) + 8), dict(N=0), dict(N=12), dict(K=0), dict(K=20), dict(K=-8), dict(act=5), dict(act=-1), dict(y_dtype=2), dict(dx_dtype=3),
                dict(dw_dtype=-1), dict(flags=4), dict(p=2.0), dict(p=float("nan")), dict(p=0.5), dict(p=0.5, rng=ODD), dict(ldx=56), dict(ldx=68),
                dict(ldx=-64), dict(ldr=16), dict(ldy=25), dict(ldz=12), dict(lddy=4), dict(lddx=60), dict(ldx=1 << 40), dict(x=None), dict(w=None),
                dict(y=None), dict(ws=None), dict(x=ODD), dict(w=ODD), dict(b=ODD), dict(r=ODD), dict(y=ODD), dict(z=ODD), dict(ws=AT + 128),
                dict(r=2 * AT, ldr=32)]:
        assert call(**bad) == 1, bad
    assert call(n=0) == 3
    assert call(M=0, x=None, y=None, ws=None) == 0
    assert f(None, AT, AT, None, None, None, AT, None, AT, 1 << 20, None) == 1


def test_linear_backward(rr):
    f = rr.lib().rr_linear_bwd
    ok = dict(dy=AT, x=AT, w=AT, z=None, rng=None, dx=2 * AT, dw=3 * AT, db=None, ws=AT, n=1 << 30)

    def call(**kw):
        a = {**ok, **kw}
        return f(C.byref(_linear(rr, **kw)), a["dy"], a["x"], a["w"], a["z"], a["rng"], a["dx"], a["dw"], a["db"], a["ws"], a["n"], None)
    for bad in [dict(dy=None), dict(x=None), dict(w=None), dict(act=1), dict(ws=None), dict(dy=ODD), dict(x=ODD), dict(w=ODD), dict(act=1, z=ODD),
                dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(ws=AT + 16), dict(p=0.1), dict(M=-3), dict(K=4), dict(lddx=32), dict(lddy=8)]:
        assert call(**bad) == 1, bad
    assert call(n=256) == 3
    assert call(M=0, dx=None, dw=None) == 0


def test_balance(rr):
    f, b, n = rr.lib().rr_balance_fwd, rr.lib().rr_balance_bwd, C.c_size_t(0)
    ok = dict(T=16, E=8, k=2, st=3, S=4, a=AT, t=AT, l=None, loss=AT, c=AT, n=AT, P=AT, ws=AT, by=1 << 20)

    def call(**kw):
        a = {**ok, **kw}
        return f(a["T"], a["E"], a["k"], a["st"], a["S"], a["a"], a["t"], a["l"], 0.1, 0.1, a["loss"], a["c"], a["n"], a["P"], a["ws"], a["by"], None)
    for bad in [dict(T=-4), dict(T=15), dict(E=0), dict(E=257), dict(k=0), dict(k=9, st=9), dict(st=1), dict(S=0), dict(S=-1), dict(a=None), dict(t=None),
                dict(loss=None), dict(c=None), dict(n=None), dict(P=None), dict(ws=None), dict(a=ODD), dict(ws=AT + 64)]:
        assert call(**bad) == 1, bad
    assert call(by=256) == 3
    for a in [(-4, 8, 2, 4, AT, AT, AT, AT), (15, 8, 2, 4, AT, AT, AT, AT), (16, 0, 2, 4, AT, AT, AT, AT), (16, 8, 9, 4, AT, AT, AT, AT),
              (16, 8, 2, 4, None, AT, AT, AT), (16, 8, 2, 4, AT, None, AT, AT), (16, 8, 2, 4, AT, AT, None, AT), (16, 8, 2, 4, AT, AT, AT, ODD)]:
        T, E, k, S, x, c, m, d = a
        assert b(T, E, k, S, x, c, m, None, 0.1, 0.1, 1.0, 0, d, None) == 1, a
    assert b(0, 8, 2, 4, None, None, None, None, 0.1, 0.1, 1.0, 0, None, None) == 0
    assert rr.lib().rr_balance_workspace_bytes(16, 8, 3, C.byref(n)) == 1 and rr.lib().rr_balance_workspace_bytes(16, 8, 4, None) == 1
    assert rr.lib().rr_balance_workspace_bytes(65536, 64, 1, C.byref(n)) == 0 and n.value > 256


def test_sizes(rr):
    assert rr.linear_workspace_bytes(0, 8, 8)[0] >= 256
    assert rr.linear_workspace_bytes(4096, 1024, 1024)[1] >= 256 + 2 * 4096 * 1024
    with pytest.raises(rr.RRError):
        rr.linear_workspace_bytes(4, 12, 8)


def test_without_a_device_the_calls_raise(rr):
    import torch
    if torch.cuda.is_available():
        pytest.skip("for machines without a GPU")
    x = torch.zeros(8, 64, dtype=torch.bfloat16)
    for call in (lambda: rr.linear_fwd(x, x, workspace=x), lambda: rr.dropout_fwd(x, 0.0, None),
                 lambda: rr.balance_fwd(x.float(), x[:, :2].int(), 1, 0.1, workspace=x)):
        with pytest.raises(Exception):
            call()
