"""MI355X-native inference from pruned, codebook-quantised, Huffman-coded layers.

``binding`` mirrors the C ABI declared in include/compressed_layer.h;
``workloads`` draws the seeded synthetic inputs.  The HIP library is loaded on
first use and there is no CPU fallback.
"""
from .binding import (PATH_AUTO, STATIC_SCRATCH_BYTES, PATH_MFMA_BF16, PATH_MFMA_F32, PATH_SPARSE, PATH_SPARSE_WIDE, CLError, Layer, LayerGroup, compress_layer,  # noqa: F401
                      compressed_conv_forward, compressed_fc_forward, compressed_fc_forward_static, compressed_fc_stack_forward, conv_block_h, conv_workspace_bytes, decode_layer,
                      fc_resolved_path, fc_stack_workspace_bytes, fc_workspace_bytes, layer_deserialize, lrn_forward, maxpool_forward, plan_batches)
from .binding import (MX_FORMS, ExpertLists, MxTensor, expert_lists, mx_dequantize, mx_experts_forward, mx_experts_resolved_form, mx_fc_forward,  # noqa: F401
                      mx_fc_resolved_form, mx_fc_workspace_bytes, mx_quantize, mx_row_blocks, route_experts)
from .binding import (F8_FORMS, F8Tensor, f8_dequantize, f8_fc_forward, f8_fc_resolved_form, f8_fc_workspace_bytes, f8_gated, f8_quantize, f8_row_blocks, f8_row_scales,  # noqa: F401
                      rms_norm)
