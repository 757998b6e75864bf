"""MI355X-native AD-PSGD worker-update engine: Python face of libadpsgd.so.

``binding`` mirrors the C ABI of include/adpsgd.h one to one; ``Engine`` adds
only what a caller needs around it: device buffers and a stream from PyTorch.
``operators`` has the operators of a worker's own training step on torch tensors.
"""
from .binding import (AdpsgdError, Handle, adpsgd_make_schedule, adpsgd_plan_rounds,  # noqa: F401
                      adpsgd_synth_gradient, adpsgd_metropolis_weights, adpsgd_verify_plan, lib, EXPORTS, LIB_PATH, MODEL_LSQ, MODEL_LOGREG,
                      MODEL_SYNTH, MODEL_MLP, MODEL_EXTERNAL, FLAG_PROFILE, FLAG_DENSE_GRADIENT, FLAG_VERIFY_PLAN, FLAG_SYNC_IN_PLACE,
                      ROUTE_AUTO, ROUTE_ROUNDS)
from .engine import Engine  # noqa: F401
from . import step_sizes  # noqa: F401

_OPERATORS = ("dense", "dense_forward", "dense_gradients", "token_log_probs", "policy_loss_and_gradient", "preference_loss_and_gradient", "AdamW",
              "distillation_loss_and_gradient", "gated", "gated_forward", "gated_gradients", "layer_norm", "layer_norm_forward", "layer_norm_gradients")


def __getattr__(name):                  # these need torch, which the host-only entry points do not
    if name in _OPERATORS:
        from . import operators
        globals().update({n: getattr(operators, n) for n in _OPERATORS})
        return globals()[name]
    raise AttributeError("module %r has no attribute %r" % (__name__, name))
