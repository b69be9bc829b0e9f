"""More of what the C entry points of the operators around the expert layer refuse before any pointer is touched (no GPU needed).
Every call below is one that has to be refused: an accepted one would launch a kernel on addresses that are not memory."""
import ctypes as C

import pytest

AT = 1 << 20                   # never dereferenced


@pytest.fixture(scope="module")
def rr():
    from paper_2402_12399_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _shape(rr, **kw):
    s = dict(M=16, N=24, K=64, act=0, y_dtype=0, dx_dtype=0, dw_dtype=0, flags=0, p=0.0, ldx=0, ldr=0, ldy=0, ldz=0, lddy=0, lddx=0)
    s.update(kw)
    return rr._CLinear(*s.values())


@pytest.mark.parametrize("which", ["ldx", "ldr", "ldy", "ldz", "lddy", "lddx"])
@pytest.mark.parametrize("pitch", [1 << 40, 1 << 60, 1 << 61, 1 << 62, (1 << 62) + 64, (1 << 63) - 64, -(1 << 62), -(1 << 63)])
def test_pitch_that_no_address_can_reach(rr, which, pitch):
    """Bytes of such a pitch do not fit into 64 bits: they wrap to 0 or to something small."""
    for dtype in (0, 1):
        s = _shape(rr, y_dtype=dtype, dx_dtype=dtype, **{which: pitch})
        assert rr.lib().rr_linear_fwd(C.byref(s), AT, 2 * AT, None, 3 * AT, None, 4 * AT, 5 * AT, 6 * AT, 1 << 30, None) == 1
        assert rr.lib().rr_linear_bwd(C.byref(s), AT, 2 * AT, 3 * AT, 4 * AT, None, 5 * AT, 6 * AT, None, 7 * AT, 1 << 30, None) == 1


@pytest.mark.parametrize("which", ["ldx", "ldr", "ldy", "ldz", "lddy", "lddx"])
def test_rows_that_no_address_can_reach(rr, which):
    """2^30 rows 2^39 bytes apart: the pitch by itself would do, the offset of the last row does not fit into 64 bits."""
    s = _shape(rr, M=1 << 30, **{which: 1 << 38})
    assert rr.lib().rr_linear_fwd(C.byref(s), AT, 2 * AT, None, 3 * AT, None, 4 * AT, 5 * AT, 6 * AT, 1 << 60, None) == 1
    assert rr.lib().rr_linear_bwd(C.byref(s), AT, 2 * AT, 3 * AT, 4 * AT, None, 5 * AT, 6 * AT, None, 7 * AT, 1 << 60, None) == 1


# Overlaps: with M, N, K = 16, 24, 64 in bf16 x and dx take 2048 bytes, W and dW 3072, y, z, residual and dy 768, bias 48; dbias 96.
APART = dict(x=AT, w=2 * AT, b=3 * AT, r=None, y=4 * AT, z=5 * AT)


@pytest.mark.parametrize("bad", [
    dict(y=AT), dict(y=2 * AT), dict(y=3 * AT - 736), dict(z=AT), dict(z=2 * AT), dict(z=3 * AT), dict(z=4 * AT), dict(r=5 * AT), dict(r=4 * AT + 16),
    dict(r=4 * AT - 16), dict(r=4 * AT, z=4 * AT), dict(y=AT + 2032), dict(y=AT - 752), dict(y=2 * AT + 3056), dict(z=4 * AT + 752), dict(z=4 * AT - 752),
    # views of one buffer: columns that meet, and a dense matrix in the gaps of a wider one that some row reaches into
    dict(y=AT + 112, ldx=128, ldy=128), dict(y=AT + 224, ldx=128, ldy=128), dict(y=AT + 16, z=AT + 256 - 16, x=6 * AT, ldy=128, ldz=128),
    dict(ldx=1024, y=AT + 2048 - 752), dict(ldx=1024, y=AT + 15 * 2048 + 112), dict(ldx=1024, y=AT + 3 * 2048 - 16),
])
def test_forward_refuses_overlaps(rr, bad):
    a = {**APART, **{k: v for k, v in bad.items() if k in APART}}
    s = _shape(rr, **{k: v for k, v in bad.items() if k not in APART})
    assert rr.lib().rr_linear_fwd(C.byref(s), a["x"], a["w"], a["b"], a["r"], None, a["y"], a["z"], 7 * AT, 1 << 30, None) == 1


@pytest.mark.parametrize("bad", [
    dict(dx=AT), dict(dx=2 * AT), dict(dx=3 * AT), dict(dx=4 * AT), dict(dw=AT), dict(dw=2 * AT), dict(dw=3 * AT), dict(dw=4 * AT), dict(dw=5 * AT),
    dict(db=AT), dict(db=2 * AT), dict(db=3 * AT), dict(db=4 * AT), dict(db=5 * AT), dict(db=6 * AT), dict(dx=AT + 752), dict(dw=2 * AT - 3056),
    dict(db=6 * AT - 80), dict(db=6 * AT + 3056), dict(dx=AT + 32, lddy=128, lddx=128), dict(dx=AT, x=None, dw=None, db=None, z=None, act=0),
    dict(dw=AT, dx=None, w=None, db=None), dict(db=AT, dx=None, dw=None, w=None, x=None, z=None, act=0)])
def test_backward_refuses_overlaps(rr, bad):
    a = dict(dy=AT, x=2 * AT, w=3 * AT, z=4 * AT, dx=5 * AT, dw=6 * AT, db=7 * AT)
    a.update({k: v for k, v in bad.items() if k in a})
    s = _shape(rr, **{"act": 1, **{k: v for k, v in bad.items() if k not in a}})
    assert rr.lib().rr_linear_bwd(C.byref(s), a["dy"], a["x"], a["w"], a["z"], None, a["dx"], a["dw"], a["db"], 8 * AT, 1 << 30, None) == 1


@pytest.mark.parametrize("xt,yt,x,r,y", [
    (1, 1, AT, None, AT + 16), (1, 1, AT + 16, None, AT), (1, 0, AT, None, AT + 384), (1, 0, AT, None, AT), (0, 1, AT, None, AT - 384),
    (0, 0, 2 * AT, AT, AT + 16), (0, 1, 2 * AT, AT + 16, AT), (1, 0, AT, AT, AT), (0, 0, AT, 2 * AT, AT - 16), (1, 1, AT, AT + 16, AT)])
def test_dropout_refuses_overlaps(rr, xt, yt, x, r, y):
    f, b = rr.lib().rr_dropout_fwd, rr.lib().rr_dropout_bwd
    assert f(100, xt, yt, x, r, 0.0, None, y, None) == 1
    if r is None:
        assert all(b(100, xt, yt, x, 0.0, None, add, y, None) == 1 for add in (0, 1))
