"""Rectify-Router MoE layer (arXiv 2402.12399) for B200: a C-ABI CUDA library
(librr.so, declared in include/rr.h) and this thin binding.

`synth` (seeded input generators) imports without the CUDA library; everything in
`binding` needs librr.so and raises if it is missing.
"""
import types

from . import synth  # noqa: F401

_BINDING = ("IR", "FR", "SCORE", "FR_SOFTMAX", "LOCAL_CAP", "GRAD_EXACT", "BF16", "F32", "RRError", "RouteTables", "alloc_tables",
            "alloc_workspace", "route_workspace_bytes", "route", "route_noalloc", "check", "moe_workspace_bytes",
            "moe_fwd", "moe_bwd", "gate_workspace_bytes", "gate_fwd", "gate_bwd", "aux_workspace_bytes",
            "aux_loss_fwd", "aux_loss_bwd", "gate_route", "gate_route_workspace_bytes", "route_loss", "route_loss_workspace_bytes", "test_set_wait_limit_ns", "Trace", "status_string", "lib",
            "LIB_PATH", "ACT_NONE", "ACT_RELU", "ACT_GELU", "ACT_GELU_TANH", "ACT_SILU", "ADD_DX", "ADD_DW", "dropout_fwd", "dropout_bwd",
            "linear_workspace_bytes", "linear_fwd", "linear_bwd", "balance_workspace_bytes", "balance_fwd", "balance_bwd",
            "NORM_LAYER", "NORM_RMS", "norm_workspace_bytes", "norm_fwd", "norm_bwd", "embed_workspace_bytes", "embed_fwd", "embed_bwd",
            "GradPlan", "grad_plan", "clip_workspace_bytes", "clip_grads")


class _Binding(types.ModuleType):
    """`binding`: a name that is set or deleted there (a wrapper, a patch in a test) is looked up anew here."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name in _BINDING:
            _kept.pop(name, None)

    def __delattr__(self, name):
        super().__delattr__(name)
        if name in _BINDING:
            _kept.pop(name, None)


_kept = globals()   # names of the binding, as attributes of this package: asking the binding each time costs a call half a microsecond


def __getattr__(name):
    if name in _BINDING or name == "binding":
        import importlib
        binding = importlib.import_module(__name__ + ".binding")
        binding.__class__ = _Binding
        if name == "binding":
            return binding   # (which the import system has made an attribute of this package)
        value = _kept[name] = getattr(binding, name)
        return value
    raise AttributeError(name)
