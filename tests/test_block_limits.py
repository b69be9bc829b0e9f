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
