"""MI355X-native multi-step speculative verification through a selective state-space layer.

The product is the C-ABI library ``libssmv.so`` (hand-written HIP for gfx950, declared in
``include/ssmv.h`` and ``include/ssmv_layers.h``); this package is its thin ctypes binding.
"""
from .binding import (  # noqa: F401
    SsmvError, ssmv_dims, ssmv_cache, ssmv_step_args, LayerCache, make_dims, load_library, LIB_PATH, EXPORTS,
    ssmv_engine_of, ssmv_stream_probe, ssmv_cache_sizes, ssmv_cache_reset, conv1d_state_update, ssm_verify_multistep, ssm_conv_verify_multistep, ssm_commit_rollback,
    ssm_commit_rollback_multi, ssm_block_multistep, ssmv_materialize_block, ssm_prefill_chunked, ssm_prefill_block, ssmv_prefill_args,
    ssmv_materialize, ssmv_first_conflict, ssmv_gated_rmsnorm, ssmv_check, ssmv_set_tuning, ssmv_copy_probe, ssmv_version,
    ssm_causal_conv, ssm_selective_scan, ssm_selective_scan_workspace, ssm_selective_step, ssmv_beam_select, ssmv_beam_workspace, ssmv_conv_history,
    ssmv_conv_args, ssmv_scan_args, ssmv_token_args, ssmv_beam_args, SSMV_BEAMS_MAX,
    SSMV_OK, SSMV_EINVAL, SSMV_EUNSUPPORTED, SSMV_EALIGN, SSMV_ESEQUENCE, SSMV_EHIP,
    SSMV_F32, SSMV_BF16, SSMV_A_SCALAR, SSMV_A_DIAG, SSMV_ACT_NONE, SSMV_ACT_SILU,
    SSMV_SNAP_BOTH, SSMV_SNAP_HJ_ONLY, SSMV_SNAP_DEFER, SSMV_WINDOW,
    SSMV_KMAX_LIMIT, SSMV_CONV_WIDTH, SSMV_CACHE_NPTR,
)
from .layers import (  # noqa: F401
    ssmv_block_norm, ssmv_block_norm_backward, ssmv_block_norm_backward_workspace, ssm_gated_recurrence, ssm_gated_recurrence_workspace,
    ssm_gated_recurrence_backward, ssm_gated_recurrence_backward_workspace, ssmv_logit_rules,
    ssmv_block_norm_args, ssmv_block_norm_grad_args, ssmv_gated_args, ssmv_gated_grad_args, ssmv_rules_args, LAYER_EXPORTS,
    SSMV_GATED_LRU, SSMV_GATED_MIX, SSMV_LAYER_STRIDE_MAX, SSMV_BLOCK_NORM_MAX, SSMV_GATED_TILE, SSMV_RULES_HISTORY_MAX, SSMV_RULES_BIAS_MAX,
)
