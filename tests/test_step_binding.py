"""What the binding itself refuses of the norm, the embedding and the clip -- shapes, types and strides, which the C entry points cannot see -- and with
which error.  CPU tensors stand in for the device's, and the library may not be called (no GPU needed)."""
import pytest
import torch


@pytest.fixture
def rr(monkeypatch):
    from paper_2402_12399_b200 import binding

    class Closed:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError(f"{name} was called")
            return call
    monkeypatch.setattr(binding, "_lib", Closed())
    monkeypatch.setattr(binding, "lib", Closed)
    monkeypatch.setattr(binding, "_here", lambda: -1)      # get_device() of a CPU tensor
    monkeypatch.setattr(binding, "_stream_of", lambda here: None)
    return binding


X, F, V, M = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8), torch.zeros(8), torch.zeros(4)
H, IDS, WS = torch.zeros(4, 8, dtype=torch.float16), torch.zeros(4, dtype=torch.int64), torch.zeros(4096, dtype=torch.uint8)


def test_a_call_that_is_right_reaches_the_library(rr):
    for name, call in (("rr_norm_fwd", lambda: rr.norm_fwd(X, V, V, residual=F, h=F.clone(), mean=M, rstd=M.clone())),
                       ("rr_norm_bwd", lambda: rr.norm_bwd(X, F, V, M, M, dh=X, dx=X.clone(), dw=V, dbias=V.clone(), workspace=WS)),
                       ("rr_embed_fwd", lambda: rr.embed_fwd(IDS, X, workspace=WS)), ("rr_embed_bwd", lambda: rr.embed_bwd(IDS, X, F, workspace=WS)),
                       ("rr_grad_plan_bytes", lambda: rr.grad_plan([X, F]))):
        with pytest.raises(AssertionError, match=name + " was called"):
            call()


@pytest.mark.parametrize("kind,says,call", [
    (TypeError, "float16", lambda r: r.norm_fwd(H)),
    (TypeError, "float16", lambda r: r.norm_fwd(X, out=H)),
    (TypeError, "float16", lambda r: r.norm_fwd(X, residual=H)),
    (TypeError, "float16", lambda r: r.norm_fwd(X, V.half())),
    (TypeError, "weight is torch.float32, bias torch.bfloat16", lambda r: r.norm_fwd(X, V, V.bfloat16())),
    (TypeError, "residual is torch.bfloat16, h torch.float32", lambda r: r.norm_fwd(X, residual=X, h=F)),
    (TypeError, "mean", lambda r: r.norm_fwd(X, mean=M.double())),
    (TypeError, "rstd", lambda r: r.norm_fwd(X, rstd=M.bfloat16())),
    (TypeError, "weight", lambda r: r.norm_fwd(X, torch.zeros(16)[::2])),
    (ValueError, "needs a residual", lambda r: r.norm_fwd(X, h=X)),
    (ValueError, "weight has shape", lambda r: r.norm_fwd(X, V[:4])),
    (ValueError, "bias has shape", lambda r: r.norm_fwd(X, V, F)),
    (ValueError, "mean has shape", lambda r: r.norm_fwd(X, mean=M[:3])),
    (ValueError, "rstd has shape", lambda r: r.norm_fwd(X, rstd=V)),
    (ValueError, "residual", lambda r: r.norm_fwd(X, residual=X[:3])),
    (ValueError, "out", lambda r: r.norm_fwd(X, out=X[:, :7])),
    (ValueError, "h", lambda r: r.norm_fwd(X, residual=X, h=X[:, :7])),
    (ValueError, "x", lambda r: r.norm_fwd(torch.zeros(8, 4).t())),
    (TypeError, "dh is torch.float32, dx torch.bfloat16", lambda r: r.norm_bwd(X, X, V, M, M, dh=F, dx=X, workspace=WS)),
    (TypeError, "dw", lambda r: r.norm_bwd(X, X, V, M, M, dw=V.bfloat16(), workspace=WS)),
    (TypeError, "float16", lambda r: r.norm_bwd(H, X, V, M, M, workspace=WS)),
    (TypeError, "float16", lambda r: r.norm_bwd(X, H, V, M, M, workspace=WS)),
    (TypeError, "float16", lambda r: r.norm_bwd(X, X, V, M, M, dx=H, workspace=WS)),
    (ValueError, "h has shape", lambda r: r.norm_bwd(X, X[:3], V, M, M, workspace=WS)),
    (ValueError, "dx", lambda r: r.norm_bwd(X, X, V, M, M, dx=X[:, :7], workspace=WS)),
    (ValueError, "dh", lambda r: r.norm_bwd(X, X, V, M, M, dh=X[:3], workspace=WS)),
    (ValueError, "dbias has shape", lambda r: r.norm_bwd(X, X, V, M, M, dbias=M, workspace=WS)),
    (ValueError, "mean has shape", lambda r: r.norm_bwd(X, X, V, M[:2], M, workspace=WS)),
    (ValueError, "rstd has shape", lambda r: r.norm_bwd(X, X, V, M, M[:2], workspace=WS)),
    (TypeError, "ids", lambda r: r.embed_fwd(M, X, workspace=WS)),
    (TypeError, "ids", lambda r: r.embed_fwd(torch.zeros(8, dtype=torch.int64)[::2], X, workspace=WS)),
    (TypeError, "float16", lambda r: r.embed_fwd(IDS, H, out=X, workspace=WS)),
    (TypeError, "float16", lambda r: r.embed_fwd(IDS, X, out_dtype=torch.float16, workspace=WS)),
    (ValueError, "table must be contiguous", lambda r: r.embed_fwd(IDS, X.t(), workspace=WS)),
    (ValueError, "out has shape", lambda r: r.embed_fwd(IDS, X, out=X[:3], workspace=WS)),
    (TypeError, "ids", lambda r: r.embed_bwd(M, X, X, workspace=WS)),
    (TypeError, "float16", lambda r: r.embed_bwd(IDS, H, X, workspace=WS)),
    (TypeError, "float16", lambda r: r.embed_bwd(IDS, X, H, workspace=WS)),
    (ValueError, "dy has shape", lambda r: r.embed_bwd(IDS, X[:3], X, workspace=WS)),
    (ValueError, "dtable must be contiguous", lambda r: r.embed_bwd(IDS, X, torch.zeros(4, 16)[:, :8], workspace=WS)),
    (ValueError, "2 gradients, but 1 outputs", lambda r: r.grad_plan([X, F], out=[X])),
    (ValueError, "out has shape", lambda r: r.grad_plan([X], out=[X[:3]])),
    (ValueError, "contiguous", lambda r: r.grad_plan([X[:, ::2]])),
    (ValueError, "contiguous", lambda r: r.grad_plan([X], out=[torch.zeros(8, 4).t()])),
    (TypeError, "float16", lambda r: r.grad_plan([H])),
    (TypeError, "float16", lambda r: r.grad_plan([X], out=[H])),
])
def test_refused(rr, kind, says, call):
    with pytest.raises(kind) as e:
        call(rr)
    assert says in str(e.value), str(e.value)


@pytest.mark.parametrize("norm,kind", [(V, ValueError), (M[:2].double(), TypeError), (torch.zeros(4)[::2], TypeError)])
def test_clip_refuses_another_norm(rr, norm, kind):
    plan = rr.GradPlan([X], [X], rr._CGradSet(), WS)
    with pytest.raises(kind, match="norm"):
        rr.clip_grads(plan, 1.0, norm=norm, workspace=WS)
    with pytest.raises(AssertionError, match="rr_clip_grads was called"):
        rr.clip_grads(plan, 1.0, norm=M[:2], workspace=WS)


def test_tensors_elsewhere_are_refused(rr, monkeypatch):
    """Every tensor of a call is on the current device: the one that is not is named with where it is."""
    monkeypatch.setattr(rr, "_here", lambda: 3)
    plan = rr.GradPlan([X], [X], rr._CGradSet(), WS)
    for call in (lambda: rr.norm_fwd(X), lambda: rr.norm_bwd(X, X, V, M, M, workspace=WS), lambda: rr.embed_fwd(IDS, X, workspace=WS),
                 lambda: rr.embed_bwd(IDS, X, X, workspace=WS), lambda: rr.grad_plan([X]), lambda: rr.clip_grads(plan, 1.0, norm=M[:2], workspace=WS)):
        with pytest.raises(ValueError, match="tensor on cpu, but the call runs on the current device cuda:3"):
            call()
