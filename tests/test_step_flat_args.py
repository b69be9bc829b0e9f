"""Where gradients of parameters may lie: at any address that is a multiple of their element.  No pointer is touched (no GPU needed): what is taken has
nothing to write, the rest is refused first."""
import ctypes as C

import pytest

AT = 1 << 20      # never dereferenced


@pytest.fixture(scope="module")
def rr():
    from paper_2402_12399_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_norm_gradients(rr):
    def call(M, dw, db):
        s = rr._CNorm(M, 24, 0, 0, 0, 0, 0, 0, rr.ADD_DW, 1e-5)
        return rr.lib().rr_norm_bwd(C.byref(s), AT, 2 * AT, 3 * AT, 4 * AT, 5 * AT, None, 6 * AT, dw, db, 9 * AT, 1 << 30, None)
    for at in (4, 8, 12, 16):
        assert call(0, 7 * AT + at, 8 * AT) == 0 and call(0, 7 * AT, 8 * AT + at) == 0
    for at in (1, 2, 3, 5, 6, 7):
        for M in (0, 16):
            assert call(M, 7 * AT + at, 8 * AT) == 1 and call(M, 7 * AT, 8 * AT + at) == 1
    # they may touch each other and what is read, but not share a byte
    assert call(16, 7 * AT + 4, 7 * AT + 96) == 1 and call(16, AT + 764, 8 * AT) == 1 and call(16, 7 * AT, 7 * AT + 4) == 1


def test_embedding_gradient(rr):
    def call(n, f32, flags, dtable):
        s = rr._CEmbed(n, 100, 24, 0, f32, 0, flags, 1.0, 0)
        return rr.lib().rr_embed_bwd(C.byref(s), AT, 2 * AT, dtable, 4 * AT, 1 << 30, None)
    for f32, size in ((0, 2), (1, 4)):
        for at in range(1, 16):
            if at % size:
                assert call(16, f32, 0, 3 * AT + at) == 1 and call(16, f32, rr.ADD_DW, 3 * AT + at) == 1 and call(0, f32, 0, 3 * AT + at) == 1
        assert call(16, f32, 0, 2 * AT + 768 - size) == 1       # the last element of dy
