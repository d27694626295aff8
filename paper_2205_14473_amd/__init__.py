"""Efficient-Adam (Chen, Shen, Liu, Luo) data-parallel round on MI355X.

The work runs in ``libea.so`` (hand-written HIP kernels for gfx950 behind the
C ABI of ``include/ea.h``); this package only binds it.  ``state`` allocates
the device buffers one round needs (PyTorch provides memory and streams).
Beside the round, ``include/ea_train.h`` holds AdamW over many tensors, the
global gradient norm, and the embedding lookup with its gradient, and
``include/ea_layer.h`` layer norm, dropout, the gated linear recurrence and the
token loss with theirs.

The binding is loaded on first use of any of its names, so that the ``build``
submodule can be imported (and the library compiled) before the library
exists; using a name with no library built raises ImportError.
"""
_EXPORTS = (
    "EA_OK", "EA_ERR_ARG", "EA_ERR_ALIGN", "EA_ERR_HIP", "EA_ERR_UNSUPPORTED",
    "EA_Q_NONE", "EA_Q_SCALED_SIGN", "EA_Q_STOCH_UNIFORM", "EA_Q_DET_UNIFORM", "EA_Q_POW2", "EA_Q_TOPK", "EA_Q_RANDK",
    "EA_SCALE_L1", "EA_SCALE_L2", "EA_SCALE_MAX", "EA_ADAM_AT_SERVER", "EA_ADAM_AT_WORKER",
    "EA_SCHED_CONSTANT", "EA_SCHED_ASSUMPTION2", "EA_SCHED_STEP_DECAY", "EA_NOALLOC_SCRATCH_BYTES",
    "Quant", "Config", "Schedule", "EAError", "lib", "LIB_PATH",
    "ea_code_bits", "ea_msg_words", "ea_msg_scales", "ea_msg_bits", "ea_workspace_bytes", "ea_validate",
    "ea_last_error", "ea_state_init", "ea_worker_compress", "ea_server_aggregate_adam", "ea_server_compress",
    "ea_worker_apply", "ea_step", "ea_step_noalloc", "ea_schedule_at", "ea_step_scheduled", "ea_run", "ea_toy_workspace_bytes",
    "ea_toy_grad", "ea_toy_step",
)
# The operators beside the round (include/ea_train.h).
_TRAIN_EXPORTS = (
    "EA_F32", "EA_BF16", "EA_F16", "EA_ROUND_NEAREST", "EA_ROUND_STOCHASTIC", "EA_STATE_BLOCK",
    "Tensor", "AdamW", "Embed", "TensorList", "ea_type",
    "ea_adamw_step", "ea_adamw_step_scheduled", "ea_grad_norm", "ea_grad_norm_workspace_bytes",
    "ea_embed_lookup", "ea_embed_grad", "ea_embed_workspace_bytes",
)
# The layers' operators (include/ea_layer.h).
_LAYER_EXPORTS = (
    "EA_GATE_PLAIN", "EA_GATE_SIGMOID", "EA_RECURRENCE_BLOCK", "EA_REDUCE_MEAN", "EA_REDUCE_SUM",
    "LayerNorm", "Dropout", "Recurrence", "TokenLoss",
    "ea_layer_norm", "ea_layer_norm_grad", "ea_layer_norm_workspace_bytes", "ea_dropout", "ea_dropout_grad",
    "ea_recurrence", "ea_recurrence_grad", "ea_recurrence_states_bytes", "ea_recurrence_workspace_bytes",
    "ea_token_loss", "ea_token_loss_workspace_bytes",
)
__all__ = list(_EXPORTS + _TRAIN_EXPORTS + _LAYER_EXPORTS)


def __getattr__(name):
    if name in _EXPORTS:
        from . import _binding as module
    elif name in _TRAIN_EXPORTS:
        from . import _train as module
    elif name in _LAYER_EXPORTS:
        from . import _layer as module
    else:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    value = globals()[name] = getattr(module, name)     # found at once from now on: small calls take a few microseconds
    return value


def __dir__():
    return sorted(set(globals()) | set(_EXPORTS + _TRAIN_EXPORTS + _LAYER_EXPORTS))
