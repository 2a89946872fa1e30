"""MI355X-native layer-wise Hessian-aware quantization (hot path of the paper's layer-wise PTQ stage).

The computation lives in libonecomp.so (hand-written HIP for gfx950, C ABI in include/onecomp.h);
this package is the thin Python binding around it plus the seeded synthetic-input generator.
"""
from .binding import (  # noqa: F401
    EXPORTED_SYMBOLS,
    LIB_PATH,
    OnecompError,
    load_library,
    onecomp_accumulate_describe,
    onecomp_accumulate_workspace_bytes,
    onecomp_attention_backward,
    onecomp_attention_forward,
    onecomp_block_norm_backward,
    onecomp_block_norm_forward,
    onecomp_clip_gradients,
    onecomp_crossgram_accumulate,
    onecomp_embedding_backward,
    onecomp_embedding_forward,
    onecomp_factor_workspace_bytes,
    onecomp_hessian_accumulate,
    onecomp_hessian_factor,
    onecomp_jointq_refine,
    onecomp_jointq_workspace_bytes,
    onecomp_linear_int8,
    onecomp_mfma_rate_probe,
    onecomp_qep_target,
    onecomp_qep_workspace_bytes,
    onecomp_quantize_layer,
    onecomp_quantize_tokens,
    onecomp_quantize_workspace_bytes,
    onecomp_rtn_sensitivity,
    onecomp_rtn_sensitivity_static,
    onecomp_token_loss_backward,
    onecomp_token_loss_forward,
    onecomp_version,
    status_string,
)
