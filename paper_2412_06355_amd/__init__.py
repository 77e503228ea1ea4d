"""DendSN layer scan on AMD Instinct MI355X (gfx950).

The forward temporal scan of a layer of dendritic spiking neurons and its
surrogate-gradient backward scan, as hand-written HIP kernels behind the C ABI
of include/dendsn.h, the token-sequence operators around such layers behind
that of include/dendsn_seq.h, and the operators of a block of layers and of its
training step behind that of include/dendsn_block.h.  This package is the Python binding of that library.
"""

from .binding import (  # noqa: F401
    EXPORTS,
    LIB_PATH,
    NOALLOC_SCRATCH_BYTES,
    DendSNConfig,
    DendSNError,
    backward,
    dendsn_backward,
    dendsn_backward_noalloc,
    dendsn_bwd_workspace_bytes,
    dendsn_ckpt_bytes,
    dendsn_forward,
    dendsn_last_error,
    dendsn_status_str,
    forward,
    lib,
)
from .block import (  # noqa: F401
    BLOCK_EXPORTS,
    AdamWConfig,
    DeltaRuleConfig,
    RMSNormConfig,
    adamw,
    adamw_states,
    block_lib,
    delta_rule,
    delta_rule_backward,
    delta_rule_step,
    dendsn_adamw_step,
    dendsn_delta_backward,
    dendsn_delta_ckpt_bytes,
    dendsn_delta_forward,
    dendsn_delta_step,
    dendsn_delta_workspace_bytes,
    dendsn_norm_backward,
    dendsn_norm_backward_residual,
    dendsn_norm_forward,
    dendsn_norm_forward_e4m3,
    dendsn_norm_workspace_bytes,
    rms_norm,
    rms_norm_backward,
    rms_norm_e4m3,
)
from .sequence import (  # noqa: F401
    SEQ_EXPORTS,
    EmbeddingConfig,
    GatedScanConfig,
    LinearCEConfig,
    dendsn_ce_forward,
    dendsn_ce_train,
    dendsn_ce_workspace_bytes,
    dendsn_ce_workspace_bytes_at,
    dendsn_embed_backward,
    dendsn_embed_forward,
    dendsn_embed_workspace_bytes,
    dendsn_scan_backward,
    dendsn_scan_ckpt_bytes,
    dendsn_scan_forward,
    dendsn_scan_step,
    dendsn_scan_workspace_bytes,
    dendsn_seq_last_error,
    embedding,
    embedding_backward,
    gated_scan,
    gated_scan_backward,
    gated_scan_step,
    linear_ce,
    linear_ce_train,
    seq_lib,
)
