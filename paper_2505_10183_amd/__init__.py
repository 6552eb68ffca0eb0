"""kt: per-GPU gradient bucket pack / weighted reduce / unpack for MI355X.

The work is done by libkt.so (hand-written HIP for gfx950 behind a C ABI, see
include/kt.h); ``binding`` marshals arguments, ``workloads`` describes the
synthetic gradient sets.
"""
from . import binding, workloads  # noqa: F401
from .binding import (Plan, KtError, kt_plan_shares, kt_plan_group_weights, kt_replan_shares,  # noqa: F401
                      kt_sampler_epoch)


def __getattr__(name):
    # The operators take torch tensors: torch is imported with the first use of one, not with the package.
    if name == "ops" or name in _OPERATORS:
        import importlib
        ops = importlib.import_module(".ops", __name__)
        globals().update({n: getattr(ops, n) for n in _OPERATORS}, ops=ops)
        return globals()[name]
    raise AttributeError("module %r has no attribute %r" % (__name__, name))


_OPERATORS = ("kt_layernorm_fwd", "kt_layernorm_bwd", "kt_layernorm_bwd_workspace", "kt_act8_shapes", "kt_act8_save", "kt_act8_restore",
              "kt_act8_weight_grad", "kt_act8_weight_grad_workspace",
              "kt_attention_fwd", "kt_attention_bwd", "kt_attention_bwd_workspace",
              "kt_embedding_fwd", "kt_embedding_bwd", "kt_embedding_bwd_workspace",
              "kt_linear_xent_fwd", "kt_linear_xent_fwd_workspace", "kt_linear_xent_bwd", "kt_linear_xent_bwd_workspace")
