"""WpAq bipolar-INT bit-plane integer GEMM for AMD MI355X (gfx950).

An MI355X-native implementation of the arbitrary-precision integer matrix
multiply of APT-LLM (arXiv 2508.19087): signed-INT codes are converted to
bipolar-INT, split into bit-planes packed in HBM, and multiplied exactly into
an int32 result with an optional fp16 scale epilogue.  The computation lives in
hand-written HIP kernels behind the C ABI of include/apt.h (libapt.so); this
package is its Python binding.
"""
from .apt import (APT_ACT_CODES, APT_ACT_FP16, APT_DECODE_MAX_M, APT_ERR_HIP, APT_ERR_INVALID_ARG, APT_ERR_UNSUPPORTED, APT_ERR_WORKSPACE,  # noqa: F401
                  APT_OK, APT_ROUTE_AUTO, APT_ROUTE_FP4_MFMA, APT_ROUTE_FP6_MFMA, APT_ROUTE_FP8_MFMA, APT_ROUTE_INT8_MFMA, APT_ROUTE_PM1_MFMA, APT_ROUTE_XOR,
                  ROUTE_NAMES, AptError, Packed, apt_config_t, apt_gemm, apt_gemm_affine,
                  apt_gemm_workspace_bytes, apt_config_table_clear, apt_config_table_size,
                  apt_last_hip_error, apt_gemm_noalloc, apt_gemm_decode, gemm_decode,
                  apt_gemm_act, apt_gemm_act_workspace_bytes, gemm_act,
                  apt_search_config, apt_search_workspace_bytes, check,
                  apt_pack_weights, apt_packed_bytes, apt_quantize_pack_activations,
                  apt_quantize_pack_activations_fp16, apt_select_config, gemm, header_functions,
                  gemm_affine, lib, pack, quantize_pack, search_config, select_config,
                  status_string)
from .mx import (APT_TYPE_BF16, APT_TYPE_FP16, APT_TYPE_FP32, Mx4, apt_dequantize_codes, apt_mx4_bytes,  # noqa: F401
                 apt_mx4_dequantize, apt_mx4_gemm, apt_mx4_gemm_act, apt_mx4_gemm_act_workspace_bytes,
                 apt_mx4_pack, apt_mx4_quantize, apt_mx4_select, apt_mx4_unpack, apt_rmsnorm_codes,
                 apt_rmsnorm_mx4, dequantize, mx4_dequantize, mx4_gemm, mx4_gemm_act, mx4_pack, mx4_quantize,
                 mx4_unpack, mx_header_functions, rmsnorm_codes, rmsnorm_mx4)
