// mx_api.hip - the extern "C" entry points declared in include/apt_mx.h:
// argument validation and launch on the caller's stream.  Validation runs
// before any HIP call, as in api.hip.
#include <math.h>

#include "mx4.h"

namespace {

using apt::hip_status;

constexpr int kMaxK = 1 << 30;         // rows are indexed with 32-bit ints
constexpr int kMaxProductK = 1 << 24;  // a tile's operands are addressed with 32-bit offsets
// Group-steps of an operand (16 GB of codes) and tiles of a product: a launch
// takes up to 256 threads for each and holds fewer than 2^32.
constexpr int64_t kMaxUnits = (int64_t)1 << 23;

bool type_ok(int t) { return t == APT_TYPE_FP16 || t == APT_TYPE_BF16 || t == APT_TYPE_FP32; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t type_bytes(int t) { return t == APT_TYPE_FP32 ? 4 : 2; }

// An operand's sizes and address.
apt_status_t operand_check(int rows, int K, const void* mx) {
  if (rows < 1 || K < 1 || mx == nullptr || !aligned(mx, 16)) return APT_ERR_INVALID_ARG;
  if (K > kMaxK || apt::mx4::groups(rows) * apt::mx4::steps(K) > kMaxUnits) return APT_ERR_UNSUPPORTED;
  return APT_OK;
}

// Rows of `type` elements in memory.
bool rows_ok(const void* x, int type, int K, int64_t stride) {
  return type_ok(type) && x != nullptr && aligned(x, type_bytes(type)) && stride >= K;
}

// The output and, where the sizes are sound, the launch.
apt_status_t product_check(int M, int N, int K, const void* w_mx, int type, const void* c) {
  const apt_status_t st = operand_check(N, K, w_mx);
  if (M < 1 || st == APT_ERR_INVALID_ARG || !type_ok(type) || c == nullptr || !aligned(c, type_bytes(type)))
    return APT_ERR_INVALID_ARG;
  if (st != APT_OK || K > kMaxProductK || apt::mx4::groups(M) * apt::mx4::steps(K) > kMaxUnits ||
      apt::mx4::gemm_tiles(M, N, K) > kMaxUnits)
    return APT_ERR_UNSUPPORTED;
  return APT_OK;
}

// Sizes of a product that an entry point takes.
bool sizes_ok(int M, int N, int K) {
  return M >= 1 && N >= 1 && K >= 1 && K <= kMaxProductK && apt::mx4::groups(M) * apt::mx4::steps(K) <= kMaxUnits &&
         apt::mx4::groups(N) * apt::mx4::steps(K) <= kMaxUnits && apt::mx4::gemm_tiles(M, N, K) <= kMaxUnits;
}

// The arguments that both norms have.
apt_status_t norm_check(int M, int K, int type, const void* x, int64_t x_stride, const void* residual,
                        int64_t residual_stride, const void* gain, double eps, const void* h, const void* y) {
  if (M < 1 || K < 1 || (type != APT_TYPE_FP16 && type != APT_TYPE_BF16)) return APT_ERR_INVALID_ARG;
  if (!rows_ok(x, type, K, x_stride)) return APT_ERR_INVALID_ARG;
  if (residual != nullptr && !rows_ok(residual, type, K, residual_stride)) return APT_ERR_INVALID_ARG;
  if (!(eps >= 0.0) || !isfinite(eps)) return APT_ERR_INVALID_ARG;
  if (!aligned(gain, 2) || !aligned(h, 2) || !aligned(y, 2)) return APT_ERR_INVALID_ARG;
  if (h != nullptr && ((h == x && x_stride != K) || (h == residual && residual_stride != K))) return APT_ERR_INVALID_ARG;
  if (y != nullptr && (y == x || y == residual || y == h)) return APT_ERR_INVALID_ARG;
  return K > kMaxK ? APT_ERR_UNSUPPORTED : APT_OK;
}

}  // namespace

extern "C" {

size_t apt_mx4_bytes(int rows, int K) {
  if (rows < 1 || K < 1) return 0;
  return apt::mx4::operand_bytes(rows, K);
}

apt_status_t apt_mx4_quantize(const void* x, int type, int rows, int K, int64_t stride, void* mx, void* stream) {
  const apt_status_t st = operand_check(rows, K, mx);
  if (st == APT_ERR_INVALID_ARG || !rows_ok(x, type, K, stride)) return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  return hip_status(apt::mx4::launch_quantize(x, type, rows, K, stride, apt::mx4::operand(mx, rows, K),
                                              static_cast<hipStream_t>(stream)));
}

apt_status_t apt_mx4_dequantize(const void* mx, int rows, int K, int type, void* out, void* stream) {
  const apt_status_t st = operand_check(rows, K, mx);
  if (st == APT_ERR_INVALID_ARG || !rows_ok(out, type, K, K)) return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  return hip_status(apt::mx4::launch_dequantize(apt::mx4::operand(mx, rows, K), rows, K, type, out,
                                                static_cast<hipStream_t>(stream)));
}

apt_status_t apt_mx4_pack(const uint8_t* codes, const uint8_t* scales, int rows, int K, void* mx, void* stream) {
  const apt_status_t st = operand_check(rows, K, mx);
  if (st == APT_ERR_INVALID_ARG || codes == nullptr || scales == nullptr) return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  return hip_status(apt::mx4::launch_pack(codes, scales, rows, K, apt::mx4::operand(mx, rows, K),
                                          static_cast<hipStream_t>(stream)));
}

apt_status_t apt_mx4_unpack(const void* mx, int rows, int K, uint8_t* codes, uint8_t* scales, void* stream) {
  const apt_status_t st = operand_check(rows, K, mx);
  if (st == APT_ERR_INVALID_ARG || codes == nullptr || scales == nullptr) return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  return hip_status(apt::mx4::launch_unpack(apt::mx4::operand(mx, rows, K), rows, K, codes, scales,
                                            static_cast<hipStream_t>(stream)));
}

apt_status_t apt_mx4_gemm(int M, int N, int K, const void* a_mx, const void* w_mx, int type, void* c, void* stream) {
  const apt_status_t st = product_check(M, N, K, w_mx, type, c);
  if (st == APT_ERR_INVALID_ARG || a_mx == nullptr || !aligned(a_mx, 16)) return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  return hip_status(apt::mx4::launch_gemm(M, N, K, apt::mx4::operand(a_mx, M, K), apt::mx4::operand(w_mx, N, K), type, c,
                                          static_cast<hipStream_t>(stream)));
}

apt_status_t apt_mx4_select(int M, int N, int K, int* rows, int* columns) {
  if (M < 1 || N < 1 || K < 1 || rows == nullptr || columns == nullptr) return APT_ERR_INVALID_ARG;
  if (!sizes_ok(M, N, K)) return APT_ERR_UNSUPPORTED;
  apt::mx4::gemm_block(M, N, K, rows, columns);
  return APT_OK;
}

size_t apt_mx4_gemm_act_workspace_bytes(int M, int N, int K) {
  if (!sizes_ok(M, N, K) || apt::mx4::gemm_prefers_rows(M, N, K)) return 0;
  return apt::mx4::operand_bytes(M, K);
}

apt_status_t apt_mx4_gemm_act(int M, int N, int K, const void* x, int x_type, int64_t x_stride, const void* w_mx,
                              int type, void* c, void* workspace, size_t workspace_bytes, void* stream) {
  const apt_status_t st = product_check(M, N, K, w_mx, type, c);
  if (st == APT_ERR_INVALID_ARG || !rows_ok(x, x_type, K, x_stride)) return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const apt::mx4::Operand w = apt::mx4::operand(w_mx, N, K);
  const size_t need = apt_mx4_gemm_act_workspace_bytes(M, N, K);
  const bool short_of_space = workspace == nullptr || workspace_bytes < need;
  if (need == 0 || (apt::mx4::gemm_takes_rows(M, K) && (short_of_space || !aligned(workspace, 16))))
    return hip_status(apt::mx4::launch_gemm_rows(M, N, K, x, x_type, x_stride, w, type, c, s));
  if (short_of_space) return APT_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return APT_ERR_INVALID_ARG;
  const apt::mx4::Operand a = apt::mx4::operand(workspace, M, K);
  const hipError_t e = apt::mx4::launch_quantize(x, x_type, M, K, x_stride, a, s);
  if (e != hipSuccess) return hip_status(e);
  return hip_status(apt::mx4::launch_gemm(M, N, K, a, w, type, c, s));
}

apt_status_t apt_rmsnorm_codes(int M, int K, int type, const void* x, int64_t x_stride, const void* residual,
                               int64_t residual_stride, const void* gain, double eps, int q, void* h, void* y,
                               int8_t* codes, uint16_t* scale, void* stream) {
  const apt_status_t st = norm_check(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y);
  if (st == APT_ERR_INVALID_ARG || q < 1 || q > 8 || codes == nullptr || scale == nullptr || !aligned(scale, 2))
    return APT_ERR_INVALID_ARG;
  if (st != APT_OK) return st;
  return hip_status(apt::mx4::launch_rmsnorm(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y, q,
                                             codes, scale, nullptr, static_cast<hipStream_t>(stream)));
}

apt_status_t apt_rmsnorm_mx4(int M, int K, int type, const void* x, int64_t x_stride, const void* residual,
                             int64_t residual_stride, const void* gain, double eps, void* h, void* y, void* mx,
                             void* stream) {
  const apt_status_t st = norm_check(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y);
  const apt_status_t so = operand_check(M, K, mx);
  if (st == APT_ERR_INVALID_ARG || so == APT_ERR_INVALID_ARG) return APT_ERR_INVALID_ARG;
  if (so != APT_OK) return so;
  const apt::mx4::Operand o = apt::mx4::operand(mx, M, K);
  return hip_status(apt::mx4::launch_rmsnorm(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y, 0,
                                             nullptr, nullptr, &o, static_cast<hipStream_t>(stream)));
}

apt_status_t apt_dequantize_codes(const int8_t* codes, const uint16_t* scale, int M, int K, int type, void* out,
                                  void* stream) {
  if (M < 1 || K < 1 || codes == nullptr || scale == nullptr || !aligned(scale, 2) || !rows_ok(out, type, K, K))
    return APT_ERR_INVALID_ARG;
  if (K > kMaxK) return APT_ERR_UNSUPPORTED;
  return hip_status(apt::mx4::launch_dequantize_codes(codes, scale, M, K, type, out, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
