"""MI355X-native hot path of Multilevel Monte Carlo gradient compression (arXiv 2507.05508):
HIP kernels for gfx950 behind a C ABI (include/mlmc.h), with a thin ctypes binding."""
from .binding import (  # noqa: F401
    MLMC_BF16, MLMC_BITS, MLMC_DEV_CAPACITY, MLMC_DEV_INTERNAL, MLMC_DEV_NONFINITE, MLMC_DEV_REDONE, MLMC_F32, MLMC_TILE, MLMC_TOPK,
    MLMC_ELIMIT, MLMC_FBITS, MLMC_VBITS, MLMC_RTN, mlmc_compress_rtn, MLMC_STOPK, MLMC_STATIC_SCRATCH_BYTES, mlmc_compress_bits_static, mlmc_aggregate_update, mlmc_message_bits,
    BitsMessage, MlmcError, Plan, SparseMessage, lib, mlmc_aggregate, mlmc_compress_bits, mlmc_compress_topk,
    MLMC_ACT_GELU, MLMC_ACT_NONE, MLMC_ACT_RELU, MLMC_DEV_RANGE, MLMC_MAX_TEACHER, mlmc_distill, mlmc_distill_workspace, mlmc_layer_norm, mlmc_layer_norm_backward,
    mlmc_layer_norm_workspace, mlmc_linear, mlmc_linear_dgrad, mlmc_linear_wgrad, mlmc_linear_workspace,
    MLMC_MAX_ANSWERS, RmsNorm, TokenLogprobs, mlmc_dropout, mlmc_linear_q8, mlmc_linear_q8_workspace, mlmc_quantize, mlmc_rms_norm, mlmc_rms_norm_backward, mlmc_rms_norm_workspace,
    mlmc_token_logprobs, mlmc_token_logprobs_backward, mlmc_token_logprobs_workspace,
    mlmc_geometric_p, mlmc_level_norms, mlmc_plan, mlmc_profile_enable, mlmc_profile_get, mlmc_profile_reset,
)
