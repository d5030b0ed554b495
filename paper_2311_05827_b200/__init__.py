"""B200-native boundary-tensor codec (AccEPT bit-level compression, Sec. 3.3-3.4).

The product is the C-ABI shared library declared in ``include/accept.h``; this package holds its
CUDA sources (``csrc/``), the in-tree build step and a ctypes binding with the same names.
"""
from .binding import (  # noqa: F401
    DEV_BAD_HEADER, DEV_COPY_TIMEOUT, DEV_NONFINITE, LAYOUT_BITPLANE, LAYOUT_INTERLEAVED, RANGE_ABSMAX, RANGE_MINMAX,
    ROUND_NEAREST, ROUND_STOCHASTIC, AcceptError, MbqParams, Params, accept_bitwidth_schedule, accept_check_params,
    accept_bounds_check_report, accept_compress, accept_compress_host, accept_compress_static, accept_compressed_size, accept_decompress, accept_decompress_host,
    accept_last_device_status, accept_launch_count, accept_launch_null, accept_parse_header, accept_payload_offset,
    accept_workspace_size, new_stream_buffer, new_workspace, accept_mbq_check_params, accept_mbq_compress,
    accept_mbq_compressed_size, accept_mbq_decompress, accept_mbq_payload_offset, accept_mbq_workspace_size,
    BLOCK_ROW, BLOCK_SQUARE, DTYPE_BF16, DTYPE_F16, DTYPE_F32, FORMAT_E4M3, FORMAT_E5M2, LayerNormParams, MatmulParams,
    QuantizeParams, accept_block_check_params, accept_block_data_size, accept_block_matmul, accept_block_quantize,
    accept_block_scale_size, accept_block_workspace_size, accept_layer_norm_backward, accept_layer_norm_check_params,
    accept_layer_norm_forward, accept_layer_norm_workspace_size, accept_matmul_check_params, accept_matmul_workspace_size,
    DropoutParams, MicroMatmulParams, MicroParams, RmsNormParams, accept_dropout, accept_dropout_check_params, accept_micro_check_params,
    accept_micro_data_size, accept_micro_dequantize, accept_micro_matmul, accept_micro_matmul_check_params, accept_micro_matmul_workspace_size,
    accept_micro_quantize, accept_micro_scale_size, accept_micro_workspace_size, accept_rms_norm_backward, accept_rms_norm_check_params,
    accept_rms_norm_forward, accept_rms_norm_workspace_size,
)
