"""MI355X-native qwZ / qgZ compression path (block-wise INT8 weight and INT4
gradient quantisation with a multi-slice dequant-sum-requant reduction), as
used by the hierarchical ZeRO++ partitioning of arXiv 2501.04266.

The compute runs in the HIP library libzq.so (C ABI in include/zq.h); this
package is its Python binding.  Importing it does not need a GPU; calling a
kernel does.
"""
from ._lib import (  # noqa: F401
    LIB_PATH,
    STATUS,
    AdamWTable,
    GradTable,
    ZQError,
    adamw_states,
    adamw_step,
    adamw_table,
    embedding,
    embedding_grad,
    embedding_grad_bytes,
    gather_tables,
    grad_clip,
    grad_norm,
    grad_table,
    int4_bytes,
    int4_dequant_gemm,
    int4_dequant_gemm_bytes,
    lib,
    num_scales,
    policy_loss,
    policy_loss_bytes,
    qgz_dequantize,
    qgz_quantize,
    qgz_reduce_dequantize,
    qgz_reduce_level,
    qgz_reduce_level_gather,
    qgz_reduce_level_gather_noalloc,
    qwz_dequant_gemm,
    qwz_dequantize,
    qwz_embedding,
    qwz_quantize,
    qwz_rms_norm,
    rms_norm,
    rms_norm_grad,
    rms_norm_grad_bytes,
    token_logp,
)
