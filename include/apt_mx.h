/*
 * apt_mx.h - C ABI of the microscaled 4-bit operators and the quantizing RMS
 * norm for AMD gfx950, in the same library as apt.h (libapt.so).
 *
 * What apt.h says of pointers, streams, errors and threads holds here too:
 * device pointers are the caller's, nothing is allocated, arguments are
 * checked on the host before anything is launched, calls enqueue on `stream`
 * and return, and status codes are apt_status_t.
 *
 * The 4-bit format (MX4) is the OCP microscaling format MXFP4: the values of a
 * row are held in blocks of 32 along K, each element an E2M1 code (sign, two
 * exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives), each block with a power-of-two scale 2^(byte - 127) in a byte
 * (E8M0).  The scale byte 255 stands for NaN: every value of its block is NaN.
 *
 * MX4 operand layout.  Rows are taken in groups of 16 and K in steps of 256
 * elements: G = ceil(R / 16), S = ceil(K / 256).  The buffer holds the codes,
 * G * S * 2048 bytes, then the scale bytes, G * S * 128 bytes.  Element k of
 * row r, with g = r / 16, s = r mod 16, t = k / 256, b = (k mod 256) / 32 (its
 * block in the step) and j = k mod 32:
 *   code   low (j even) or high (j odd) nibble of byte
 *          ((g * S + t) * 8 + b) * 256 + s * 16 + j / 2
 *   scale  byte G * S * 2048 + (g * S + t) * 128 + (b mod 2) * 64 + s * 4 + b / 2
 * so that the 16 bytes of a block are one lane's operand of the block-scaled
 * MFMA, the operands of 16 rows are contiguous, and the four scales that a lane
 * needs in a step are one dword.  In rows r < R the codes and scale bytes of the
 * elements K <= k < 256 S are zero; those of rows r >= R are never read as
 * values and are left as they were.  Buffers are 16-byte aligned.
 */
#ifndef APT_MX_H
#define APT_MX_H

#include "apt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of inputs and outputs. */
enum {
  APT_TYPE_FP16 = 1,
  APT_TYPE_BF16 = 2,
  APT_TYPE_FP32 = 3
};

/* Bytes of an MX4 operand of `rows` rows of K values; 0 for rows < 1 or K < 1. */
size_t apt_mx4_bytes(int rows, int K);

/* Quantizes rows to MX4.  For each block of 32 elements (the last one of a row
 * may be shorter) with the largest magnitude m:
 *   scale = 2^e, e = floor(log2 m) - 2, at least -127 (m = 0: -127);
 *   code  = the E2M1 value nearest x / 2^e, ties to the even code, magnitudes
 *           above 6 to 6; the sign is kept, also of a zero.
 * A block that holds an infinity or a NaN gets scale byte 255 and codes 0.
 *   x       device, [rows][K] of `type`, row r at x + r * stride elements,
 *           aligned to its element size
 *   stride  elements from a row to the next, >= K
 *   mx      device, apt_mx4_bytes(rows, K) bytes, 16-byte aligned
 * Errors: APT_ERR_INVALID_ARG for rows < 1, K < 1, stride < K, an unknown type,
 * NULL or misaligned pointers; APT_ERR_UNSUPPORTED for K > 2^30 or an operand
 * of more than 2^23 groups x steps (16 GB); APT_ERR_HIP on launch failure. */
apt_status_t apt_mx4_quantize(const void* x, int type, int rows, int K, int64_t stride, void* mx,
                              void* stream);

/* The values of an MX4 operand, row-major [rows][K] of `type` (rounded to
 * nearest even for fp16; exact for bf16 and fp32; infinite past the type's range,
 * in bf16 and fp32 some values of the scale bytes 253 and 254, which quantizing
 * does not give).
 *   out  device, aligned to its element size
 * Errors as apt_mx4_quantize. */
apt_status_t apt_mx4_dequantize(const void* mx, int rows, int K, int type, void* out, void* stream);

/* Lays row-major MX4 data (as checkpoints store it) out as an operand, and back.
 *   codes   device, [rows][ceil(K / 2)] bytes: element k in byte k / 2, the even
 *           element in the low nibble
 *   scales  device, [rows][ceil(K / 32)] scale bytes
 * Packing ignores what the codes hold behind K; unpacking writes 0 there.
 * Errors as apt_mx4_quantize (codes and scales need no alignment). */
apt_status_t apt_mx4_pack(const uint8_t* codes, const uint8_t* scales, int rows, int K, void* mx,
                          void* stream);
apt_status_t apt_mx4_unpack(const void* mx, int rows, int K, uint8_t* codes, uint8_t* scales,
                            void* stream);

/* C = A * W^T of two MX4 operands, C[m][n] = sum_k A[m][k] W[n][k], with fp32
 * sums and one rounding (to nearest even) to the output's type.
 *   a_mx, w_mx  device, MX4 operands of M and N rows of K values
 *   type, c     output type and device [M][N] row-major, aligned to its element size
 * The result does not depend on what else runs: sums are taken in an order fixed
 * by the sizes.  NaN scales reach only the outputs of their rows.
 * Errors: APT_ERR_INVALID_ARG for sizes < 1, an unknown type, NULL or misaligned
 * pointers; APT_ERR_UNSUPPORTED for K > 2^24, an operand of more than 2^23
 * groups x steps or an output of more than 2^23 tiles; APT_ERR_HIP on launch
 * failure. */
apt_status_t apt_mx4_gemm(int M, int N, int K, const void* a_mx, const void* w_mx, int type, void* c,
                          void* stream);

/* The kernel that apt_mx4_gemm takes for a problem, by the block of outputs that
 * one of its workgroups makes: 16 x 16, 32 x 16, 32 x 32 or 64 x 32 (the few-row
 * kernel), or 32 x 128, 64 x 128, 128 x 128, 128 x 256 or 256 x 256 (tiles).  It
 * depends on the sizes alone.  (apt_mx4_gemm_act without a workspace is the few-row
 * kernel in blocks of 16 x 16 as well.)
 *   rows, columns  host, receive the block
 * Errors: APT_ERR_INVALID_ARG for sizes < 1 or NULL pointers; APT_ERR_UNSUPPORTED
 * as apt_mx4_gemm. */
apt_status_t apt_mx4_select(int M, int N, int K, int* rows, int* columns);

/* C = A * W^T with the activations given unpacked and quantized inside the call
 * as apt_mx4_quantize does; the result equals that of apt_mx4_quantize followed
 * by apt_mx4_gemm, bit for bit.  Up to 16 rows of together 16384 elements (rows
 * padded to 256) can be quantized by the product's kernel itself, which needs no
 * workspace; from three rows on, where these elements times N / 16 are more than
 * 2^24, quantizing them into a workspace first is faster, and is done where there
 * is one.  Other rows need it.
 *   x, x_type, x_stride  as apt_mx4_quantize, M rows
 *   workspace, workspace_bytes  device scratch of at least
 *               apt_mx4_gemm_act_workspace_bytes(M, N, K) bytes, 16-byte aligned
 *               (ignored when 0); overwritten; calls sharing it must not overlap in time
 * Errors as apt_mx4_quantize and apt_mx4_gemm, and APT_ERR_WORKSPACE when a
 * workspace that is needed is missing or too small. */
size_t apt_mx4_gemm_act_workspace_bytes(int M, int N, int K);
apt_status_t apt_mx4_gemm_act(int M, int N, int K, const void* x, int x_type, int64_t x_stride,
                              const void* w_mx, int type, void* c, void* workspace,
                              size_t workspace_bytes, void* stream);

/* RMS norm of rows, with the residual's addition in front and the operand of a
 * quantized product behind.  With T the inputs' type (fp16 or bf16), per row:
 *   h    = T(x + residual) (x itself without a residual)
 *   f    = fp32(1 / sqrt(sum_k h[k]^2 / K + eps)), the sum and its root in fp64
 *   y[k] = T(fp32(fp32(h[k] * f) * gain[k])) (fp32(h[k] * f) without a gain)
 * The fp64 value is good to a few parts in 2^50, whatever order the row is summed
 * in: y and its codes follow the definition unless it lies that close to a border
 * between two fp32 roundings, where f may be the neighbour.  apt_rmsnorm_codes then
 * quantizes the row to q-bit codes, 1 <= q <= 8, by the rule of
 * apt_quantize_pack_activations_fp16:
 *   scale = fp16(fp32(max_k |y[k]| / (2^q - 1)))
 *   code  = floor(y[k] / (2 scale)), in [-2^(q-1), 2^(q-1) - 1], value
 *           (2 code + 1) scale; 0 where the scale is 0
 * as apt_gemm_act and apt_gemm_decode take them (APT_ACT_CODES with a_scale); a
 * row whose y holds a NaN or an infinity, or whose scale would be infinite, gets
 * a NaN scale and codes 0.  apt_rmsnorm_mx4 quantizes y as apt_mx4_quantize does.
 *   type       APT_TYPE_FP16 or APT_TYPE_BF16, of x, residual, gain, h and y alike
 *   x, residual  device, M rows of K with their strides in elements (>= K);
 *              residual NULL for none (its stride is then ignored)
 *   gain       device [K] or NULL
 *   eps        >= 0 and finite
 *   h          device [M][K] row-major or NULL: receives h; it may be x or
 *              residual itself where that one's stride is K, and overlaps
 *              nothing else
 *   y          device [M][K] row-major or NULL: receives y; overlaps nothing else
 *   codes, scale  device int8 [M][K] and fp16 bits [M]
 *   mx         device, apt_mx4_bytes(M, K) bytes, 16-byte aligned
 * Errors: APT_ERR_INVALID_ARG for sizes < 1, q outside [1, 8], a stride < K, a
 * type other than the two, a negative or non-finite eps, NULL x, codes, scale or
 * mx, a y that is x, residual or h, or misaligned pointers; APT_ERR_UNSUPPORTED
 * for K > 2^30; APT_ERR_HIP. */
apt_status_t apt_rmsnorm_codes(int M, int K, int type, const void* x, int64_t x_stride,
                               const void* residual, int64_t residual_stride, const void* gain,
                               double eps, int q, void* h, void* y, int8_t* codes, uint16_t* scale,
                               void* stream);
apt_status_t apt_rmsnorm_mx4(int M, int K, int type, const void* x, int64_t x_stride,
                             const void* residual, int64_t residual_stride, const void* gain,
                             double eps, void* h, void* y, void* mx, void* stream);

/* The values (2 code + 1) scale that codes with a scale per row stand for, row-
 * major [M][K] of `type`, rounded once.
 *   codes, scale  device int8 [M][K] and fp16 bits [M], as apt_rmsnorm_codes
 * Errors: APT_ERR_INVALID_ARG for sizes < 1, an unknown type, NULL or misaligned
 * pointers; APT_ERR_UNSUPPORTED for K > 2^30; APT_ERR_HIP. */
apt_status_t apt_dequantize_codes(const int8_t* codes, const uint16_t* scale, int M, int K, int type,
                                  void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* APT_MX_H */
