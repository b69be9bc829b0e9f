"""What the C entry points of the norm, the embedding and the clip refuse, before any pointer is touched (no GPU needed).  Every call that is
expected to be refused would launch a kernel on addresses that are not memory if it were not."""
import ctypes as C

import pytest

AT, ODD = 1 << 20, (1 << 20) + 8      # never dereferenced


@pytest.fixture(scope="module")
def rr():
    from paper_2402_12399_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _norm(rr, **kw):
    s = dict(M=16, N=24, kind=0, x_dtype=0, h_dtype=0, w_dtype=0, y_dtype=0, dx_dtype=0, flags=0, eps=1e-5, ldx=0, ldr=0, ldh=0, ldy=0, lddy=0, lddh=0, lddx=0)
    s.update({k: v for k, v in kw.items() if k in s})
    return rr._CNorm(*s.values())


SHAPES = [dict(M=-1), dict(N=0), dict(N=-8), dict(N=32769), dict(kind=2), dict(kind=-1), dict(x_dtype=2), dict(h_dtype=-1), dict(w_dtype=3), dict(y_dtype=2),
          dict(dx_dtype=2), dict(flags=1), dict(flags=4), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf"))] + \
    [{ld: v} for ld in ("ldx", "ldr", "ldh", "ldy", "lddy", "lddh", "lddx") for v in (23, -24, 1 << 40, 1 << 62, (1 << 63) - 24, -(1 << 63))]


def test_norm_forward(rr):
    ok = dict(x=AT, r=None, w=2 * AT, b=None, h=None, y=3 * AT, m=None, s=None)

    def call(**kw):
        a = {**ok, **kw}
        return rr.lib().rr_norm_fwd(C.byref(_norm(rr, **kw)), a["x"], a["r"], a["w"], a["b"], a["h"], a["y"], a["m"], a["s"], None)
    # (16 x 24 in bf16 are 768 bytes, 48 a row; the vectors 48 and 64)
    for bad in SHAPES + [dict(x=None), dict(y=None), dict(x=ODD), dict(r=ODD), dict(w=ODD), dict(b=ODD), dict(y=ODD), dict(m=ODD), dict(s=ODD),
                         dict(h=4 * AT), dict(r=4 * AT, h=ODD), dict(kind=1, m=4 * AT), dict(y=AT + 16), dict(y=AT - 16), dict(y=AT, y_dtype=1),
                         dict(y=AT, ldx=32), dict(y=2 * AT), dict(b=3 * AT), dict(r=4 * AT, h=3 * AT), dict(r=4 * AT, h=3 * AT + 752), dict(r=4 * AT, h=AT, x_dtype=1),
                         dict(r=4 * AT, y=4 * AT + 32), dict(r=4 * AT, y=4 * AT, y_dtype=1), dict(m=AT), dict(s=AT + 704), dict(m=3 * AT), dict(s=3 * AT),
                         dict(m=5 * AT, s=5 * AT), dict(m=5 * AT, s=5 * AT + 48), dict(s=2 * AT), dict(m=4 * AT, r=4 * AT), dict(r=4 * AT, h=2 * AT),
                         dict(r=4 * AT, h=4 * AT, ldr=32)]:
        assert call(**bad) == 1, bad
    assert call(M=0, x=None, y=None) == 0
    assert rr.lib().rr_norm_fwd(None, AT, None, None, None, None, 2 * AT, None, None, None) == 1


def test_norm_backward(rr):
    ok = dict(dy=AT, h=2 * AT, w=3 * AT, m=4 * AT, s=5 * AT, dh=None, dx=6 * AT, dw=7 * AT, db=8 * AT, ws=9 * AT, n=1 << 30)

    def call(**kw):
        a = {**ok, **kw}
        return rr.lib().rr_norm_bwd(C.byref(_norm(rr, **kw)), a["dy"], a["h"], a["w"], a["m"], a["s"], a["dh"], a["dx"], a["dw"], a["db"], a["ws"], a["n"], None)
    for bad in SHAPES + [dict(dy=None), dict(h=None), dict(m=None), dict(s=None), dict(ws=None), dict(ws=9 * AT + 128), dict(dy=ODD), dict(h=ODD), dict(w=ODD),
                         dict(m=ODD), dict(s=ODD), dict(dh=ODD), dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(dx=AT + 16), dict(dx=AT, dx_dtype=1),
                         dict(dx=2 * AT, lddx=32), dict(dx=3 * AT), dict(dx=4 * AT), dict(dx=5 * AT), dict(dx=7 * AT), dict(dw=AT), dict(dw=2 * AT), dict(dw=3 * AT),
                         dict(dw=4 * AT), dict(db=5 * AT), dict(db=7 * AT), dict(db=7 * AT + 80), dict(db=6 * AT + 752), dict(dh=10 * AT, dx=10 * AT + 768 - 16),
                         dict(dh=10 * AT, dw=10 * AT)]:
        assert call(**bad) == 1, bad
    assert call(n=256) == 3
    assert call(M=0, dy=None, dw=None, db=None) == 0
    assert call(dx=None, dw=None, db=None) == 0         # nothing is wanted
    n = C.c_size_t(0)
    assert rr.lib().rr_norm_workspace_bytes(4, 0, C.byref(n)) == 1 and rr.lib().rr_norm_workspace_bytes(-1, 8, C.byref(n)) == 1
    assert rr.lib().rr_norm_workspace_bytes(4, 8, None) == 1
    assert rr.lib().rr_norm_workspace_bytes(4096, 1024, C.byref(n)) == 0 and n.value >= 256 + 2 * 4096


def _embed(rr, **kw):
    s = dict(n=16, V=100, d=24, wide_ids=0, table_dtype=0, y_dtype=0, flags=0, scale=1.0, ldy=0)
    s.update({k: v for k, v in kw.items() if k in s})
    return rr._CEmbed(*s.values())


def test_embedding(rr):
    def calls(**kw):
        a = {**dict(ids=AT, i=2 * AT, o=3 * AT, ws=4 * AT, by=1 << 30), **kw}
        return [f(C.byref(_embed(rr, **kw)), a["ids"], a["i"], a["o"], a["ws"], a["by"], None) for f in (rr.lib().rr_embed_fwd, rr.lib().rr_embed_bwd)]
    # (ids 64 bytes, 16 x 24 in bf16 768, the table 4800)
    for bad in [dict(n=-1), dict(n=(1 << 30) + 1), dict(V=0), dict(V=-1), dict(V=(1 << 30) + 1), dict(d=0), dict(d=(1 << 26) + 1, V=1), dict(V=1 << 20, d=1 << 20),
                dict(wide_ids=2), dict(wide_ids=-1), dict(table_dtype=2), dict(y_dtype=-1), dict(flags=1), dict(flags=6), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(scale=float("-inf")), dict(ldy=23), dict(ldy=-24), dict(ldy=1 << 40), dict(ldy=1 << 62), dict(ldy=-(1 << 63)),
                dict(n=1 << 30, ldy=1 << 38), dict(ids=None), dict(i=None), dict(o=None), dict(ws=None), dict(ids=AT + 2), dict(ids=AT + 4, wide_ids=1), dict(i=ODD),
                dict(o=ODD), dict(ws=4 * AT + 128), dict(o=2 * AT), dict(o=2 * AT + 752), dict(o=AT), dict(o=AT + 48), dict(i=3 * AT - 752)]:
        assert calls(**bad) == [1, 1], bad
    assert calls(by=255) == [3, 3]
    assert calls(n=0, ids=None, i=None, o=None, ws=None) == [0, 1]      # (backward there is a table to set to zero)
    assert calls(n=0, flags=2, o=None)[1] == 0
    a, b = C.c_size_t(0), C.c_size_t(0)
    f = rr.lib().rr_embed_workspace_bytes
    assert f(-1, 8, 8, C.byref(a), C.byref(b)) == 1 and f(8, 0, 8, C.byref(a), C.byref(b)) == 1 and f(8, 8, 0, C.byref(a), None) == 1
    assert f(1 << 30, 1 << 30, 1, C.byref(a), C.byref(b)) == 0 and a.value == 256 and b.value > (1 << 30) * 8
    assert f(0, 8, 8, None, None) == 0


def _grads(rr, *items):
    out = (rr._CGrad * max(1, len(items)))()
    for c, g in zip(out, items):
        c.src, c.dst, c.n, c.src_dtype, c.dst_dtype = g
    return out


def test_plan(rr):
    s, n = rr._CGradSet(), C.c_size_t(0)

    def call(*items, tensors=None, plan=AT, by=1 << 20, out=s):
        return rr.lib().rr_grad_plan(len(items) if tensors is None else tensors, _grads(rr, *items), plan, by, C.byref(out) if out else None, None)
    A, B = 1 << 30, 1 << 31
    for bad in [[(A, A, -1, 0, 0)], [(0, A, 4, 0, 0)], [(A + 1, A + 1, 4, 0, 0)], [(A + 2, A + 2, 4, 1, 1)], [(A, B + 2, 4, 0, 1)], [(A, A, 4, 2, 2)], [(A, B, 4, 0, 2)],
                [(A, A, 4, 0, 1)], [(A, A, 4, 1, 0)], [(A, A + 4, 4, 1, 1)], [(A, A - 8, 4, 0, 1)], [(A, None, 1 << 42, 0, 0)],
                [(A, None, 1 << 41, 0, 0), (A, None, 1 << 41, 0, 0)],
                [(A, A, 8, 0, 0), (A, A, 8, 0, 0)], [(A, A, 8, 0, 0), (A + 14, A + 14, 8, 0, 0)], [(A, None, 8, 0, 0), (A + 14, None, 8, 0, 0)],
                [(A, B, 8, 0, 0), (A + 64, B + 14, 8, 0, 0)], [(A, B, 8, 1, 1), (B, A, 8, 1, 1)], [(A, B, 8, 1, 0), (B + 12, None, 8, 1, 1)],
                [((1 << 64) - 16, None, 16, 0, 0)]]:
        assert call(*bad) == 1, bad
    fine = (A, B, 8, 0, 0)
    assert call(fine, tensors=-1) == 1 and call(fine, tensors=(1 << 20) + 1) == 1
    assert call(fine, plan=None) == 1 and call(fine, plan=AT + 8) == 1 and call(fine, out=None) == 1
    assert rr.lib().rr_grad_plan(1, None, AT, 1 << 20, C.byref(s), None) == 1
    assert call(fine, by=64) == 3
    f = rr.lib().rr_grad_plan_bytes
    assert f(-1, C.byref(n)) == 1 and f((1 << 20) + 1, C.byref(n)) == 1 and f(1, None) == 1
    assert f(0, C.byref(n)) == 0 and n.value > 0 and f(1 << 20, C.byref(n)) == 0


def test_clip(rr):
    n = C.c_size_t(0)
    assert rr.lib().rr_clip_workspace_bytes(None) == 1
    assert rr.lib().rr_clip_workspace_bytes(C.byref(n)) == 0 and n.value > 256

    def call(plan=AT, tensors=1, chunk=2048, chunks=1, bound=1.0, norm=2 * AT, ws=3 * AT, by=1 << 20):
        s = rr._CGradSet(plan, tensors, chunk, chunks)
        return rr.lib().rr_clip_grads(C.byref(s), bound, norm, ws, by, None)
    for bad in [dict(plan=None), dict(plan=AT + 8), dict(tensors=-1), dict(tensors=(1 << 20) + 1), dict(chunk=0), dict(chunk=12), dict(chunks=-1), dict(bound=-1.0),
                dict(bound=float("nan")), dict(norm=None), dict(norm=2 * AT + 2), dict(ws=None), dict(ws=3 * AT + 128)]:
        assert call(**bad) == 1, bad
    assert call(by=256) == 3
    assert rr.lib().rr_clip_grads(None, 1.0, AT, AT, 1 << 20, None) == 1


def test_the_binding_says_what_is_wrong(rr):
    """Shapes and types that the C entry points cannot see are refused by the binding; without a device all of them are."""
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    f = torch.zeros(8)
    for call in (lambda: rr.norm_fwd(x), lambda: rr.norm_bwd(x, x, None, None, f[:4], kind=1, workspace=x), lambda: rr.embed_fwd(f[:2].int(), x, workspace=x),
                 lambda: rr.embed_bwd(f[:4].int(), x, x, workspace=x), lambda: rr.grad_plan([x]), lambda: rr.clip_grads([x], 1.0)):
        with pytest.raises(Exception):
            call()
    with pytest.raises(ValueError):
        rr.grad_plan([x], out=[])
