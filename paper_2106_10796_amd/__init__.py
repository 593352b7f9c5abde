"""CD-SGD per-step data-parallel hot path on MI355X (gfx950).

The product is libcdsgd.so (HIP kernels behind the C ABI in include/cdsgd.h, include/cdsgd_ops.h and
include/cdsgd_block.h);
`binding` marshals torch tensors into it, `synth` makes seeded inputs and
`runner` lays a workload out in device memory and drives the calls.
"""
from . import binding  # noqa: F401
from .binding import (AdamWPlan, BlockNorm, CdsgdError, GradNorm, Mxfp4, Mxint8, Plan, StaticLayerList, Trainer,  # noqa: F401
                      cdsgd_attention_backward, cdsgd_attention_forward, cdsgd_decode_sum, cdsgd_decode_sum_sparse, cdsgd_gated_backward,
                      cdsgd_gated_forward, cdsgd_mxfp4_dequantize, cdsgd_mxfp4_matmul, cdsgd_mxfp4_quantize, cdsgd_mxint8_dequantize,
                      cdsgd_mxint8_quantize, cdsgd_quantize_pack, cdsgd_sparse_encode, cdsgd_step_fused_static, cdsgd_update,
                      new_attention_workspace, new_block_norm_workspace, new_mxfp4, new_mxfp4_workspace, new_mxint8, new_packed, new_sparse,
                      packed_words, sparse_words, state_blocks)
