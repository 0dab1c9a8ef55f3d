// mx4.h - the MX4 operand (32-element blocks of E2M1 codes, an E8M0 scale
// byte each; layout fixed in apt_mx.h) and the conversion of one block, shared
// by the quantizer, the norm and the products, for gfx950.
#pragma once

#include "apt_internal.h"
#include "../../include/apt_mx.h"

namespace apt {
namespace mx4 {

constexpr int kBlock = 32;    // elements per scale
constexpr int kStep = 256;    // elements of K per step of the layout
constexpr int kGroup = 16;    // rows per group
constexpr int kCodeBytes = kGroup * kStep / 2;        // codes of a group and step
constexpr int kScaleBytes = kGroup * kStep / kBlock;  // scale bytes of a group and step

inline int64_t groups(int rows) { return ((int64_t)rows + kGroup - 1) / kGroup; }
inline int steps(int K) { return K / kStep + (K % kStep != 0); }  // (any int: sizes are asked for before they are checked)
inline size_t code_bytes(int rows, int K) { return (size_t)groups(rows) * steps(K) * kCodeBytes; }
inline size_t operand_bytes(int rows, int K) {
  return (size_t)groups(rows) * steps(K) * (kCodeBytes + kScaleBytes);
}

// An operand of `rows` rows in memory.
struct Operand {
  uint8_t* codes;
  uint8_t* scales;
  int64_t groups;
  int steps;
};
inline Operand operand(void* mx, int rows, int K) {
  uint8_t* p = static_cast<uint8_t*>(mx);
  return {p, p + code_bytes(rows, K), groups(rows), steps(K)};
}
inline Operand operand(const void* mx, int rows, int K) { return operand(const_cast<void*>(mx), rows, K); }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(1)));  // at any byte
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Element types.  kVec elements are one 16-byte vector of dwords.
struct Half {
  static constexpr int kBytes = 2, kVec = 8;
  static constexpr uint32_t kInf = 0x7C00u;  // magnitude bits of infinity
  __device__ static float to_float(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  __device__ static uint16_t from_float(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
  __device__ static uint32_t pair(float a, float b) {  // rounded to nearest even, a in the low half
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
  }
};
struct Bf16 {
  static constexpr int kBytes = 2, kVec = 8;
  static constexpr uint32_t kInf = 0x7F80u;
  __device__ static float to_float(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
  __device__ static uint16_t from_float(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  __device__ static uint32_t pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
  }
};
struct Float {
  static constexpr int kBytes = 4, kVec = 4;
  static constexpr uint32_t kInf = 0x7F800000u;
};

// Largest magnitude bits of a vector: of 16-bit types, a dword of two maxima
// to be folded by `widest`.
template <class T>
__device__ __forceinline__ uint32_t fold_magnitude(uint32_t m, u32x4 v) {
  if constexpr (T::kBytes == 2) {
    u16x2 r = __builtin_bit_cast(u16x2, m);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r = __builtin_elementwise_max(r, __builtin_bit_cast(u16x2, v[i] & 0x7FFF7FFFu));
    return __builtin_bit_cast(uint32_t, r);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, v[i] & 0x7FFFFFFFu);
    return m;
  }
}
template <class T>
__device__ __forceinline__ uint32_t widest(uint32_t m) {
  return T::kBytes == 2 ? max(m & 0xFFFFu, m >> 16) : m;
}

// Scale byte of a block whose largest magnitude has the bits m: the exponent
// field of m in fp32 less 2, at least 0; 255 for an infinity or a NaN.
template <class T>
__device__ __forceinline__ uint32_t scale_byte(uint32_t m) {
  if (m >= T::kInf) return 255u;
  uint32_t e;
  if constexpr (T::kBytes == 4) e = m >> 23;
  else e = __builtin_bit_cast(uint32_t, T::to_float((uint16_t)m)) >> 23;
  return max(e, 2u) - 2u;
}

// 2^(byte - 127) of a byte below 255 (byte 0 is a subnormal fp32).
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u);
}

// The eight codes (element i in nibble i) of eight elements: two vectors of
// Float, one of the others.  The conversion rounds to nearest even and
// saturates at 6.
template <class T>
__device__ __forceinline__ uint32_t codes_of(const u32x4* v, float scale) {
  uint32_t c = 0u;
  if constexpr (T::kBytes == 4) {
    // (the casts make values of the elements: a bit cast of a vector's element itself reads element 0)
    const u32x4 a = v[0], b = v[1];
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __builtin_bit_cast(float, (uint32_t)a[2]), __builtin_bit_cast(float, (uint32_t)a[3]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __builtin_bit_cast(float, (uint32_t)b[2]), __builtin_bit_cast(float, (uint32_t)b[3]), scale, 3);
  } else if constexpr (T::kInf == Half::kInf) {
    const u32x4 a = v[0];
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)a[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)a[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)a[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)a[3]), scale, 3);
  } else {
    const u32x4 a = v[0];
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)a[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)a[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)a[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)a[3]), scale, 3);
  }
  return c;
}

// One 16-byte vector of a row from element k on, at any address (as fast as an
// aligned one where neighbouring lanes read neighbouring vectors: 2048 x 4095 and
// 2048 x 4096 norms within 5%).
template <class T>
__device__ __forceinline__ u32x4 load_whole(const uint8_t* row, int k) {
  return *reinterpret_cast<const any_u32x4*>(row + (int64_t)k * T::kBytes);
}
// The same near a row's end, in two steps so that several loads leave before the
// first is waited for: load_near reads the vector, or the row's last whole one
// where it would cross the end, and settle shifts that one down and leaves zero
// bits from element K on.  (Rows shorter than a vector take element loads.)
template <class T>
__device__ __forceinline__ u32x4 load_near(const uint8_t* row, int k, int K) {
  if (K >= T::kVec) return load_whole<T>(row, min(k, K - T::kVec));
  u32x4 v = {0u, 0u, 0u, 0u};
  if constexpr (T::kBytes == 4) {
    const uint32_t* const p = reinterpret_cast<const uint32_t*>(row);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k + i < K) v[i] = p[k + i];
  } else {
    const uint16_t* const p = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < K) v[i / 2] |= (uint32_t)p[k + i] << (16 * (i % 2));
  }
  return v;
}
template <class T>
__device__ __forceinline__ u32x4 settle(u32x4 v, int k, int K) {
  const int over = k + T::kVec - K;  // elements past the end
  if (K < T::kVec || __builtin_amdgcn_ballot_w64(over > 0) == 0ull) return v;
  const uint32_t bits = (uint32_t)max(over, 0) * (8 * T::kBytes);
  // down by two dwords, one, and what is left of one (0 or 16 bits)
  u32x4 r = v;
  r = bits & 64u ? u32x4{r[2], r[3], 0u, 0u} : r;
  r = bits & 32u ? u32x4{r[1], r[2], r[3], 0u} : r;
  if constexpr (T::kBytes == 2)
    r = u32x4{__builtin_amdgcn_alignbit(r[1], r[0], bits), __builtin_amdgcn_alignbit(r[2], r[1], bits),
              __builtin_amdgcn_alignbit(r[3], r[2], bits), __builtin_amdgcn_alignbit(0u, r[3], bits)};
  return bits >= 128u ? u32x4{0u, 0u, 0u, 0u} : r;
}

// The first n (at most 16) bytes of a vector to any byte address, n a multiple of
// kBytes: whole, or as pieces of 8, 4, 2 and 1 bytes.
// kStream: whole vectors go past the L2 cache (a template's parameter: the compiler
// makes one plain store of both sides of a branch).
template <int kBytes, bool kStream = false>
__device__ __forceinline__ void store_bytes(uint8_t* dst, int n, u32x4 v) {
  typedef uint32_t any_u32x2 __attribute__((ext_vector_type(2), aligned(1)));
  typedef uint32_t any_u32 __attribute__((aligned(1)));
  typedef uint16_t any_u16 __attribute__((aligned(1)));
  if (n >= 16) {
    if (kStream) __builtin_nontemporal_store(v, reinterpret_cast<any_u32x4*>(dst));
    else *reinterpret_cast<any_u32x4*>(dst) = v;
    return;
  }
  uint64_t left = (uint64_t)v[0] | (uint64_t)v[1] << 32;
  if (n & 8) {
    *reinterpret_cast<any_u32x2*>(dst) = u32x2{v[0], v[1]};
    dst += 8;
    left = (uint64_t)v[2] | (uint64_t)v[3] << 32;
  }
  if (n & 4) {
    *reinterpret_cast<any_u32*>(dst) = (uint32_t)left;
    dst += 4;
    left >>= 32;
  }
  if (kBytes <= 2 && (n & 2)) {
    *reinterpret_cast<any_u16*>(dst) = (uint16_t)left;
    dst += 2;
    left >>= 16;
  }
  if (kBytes == 1 && (n & 1)) *dst = (uint8_t)left;
}
// A vector of a row from element k on, as far as the row goes.
template <class T, bool kStream = false>
__device__ __forceinline__ void store_vector(uint8_t* row, int k, int K, u32x4 v) {
  if (k < K) store_bytes<T::kBytes, kStream>(row + (int64_t)k * T::kBytes, (K - k < T::kVec ? K - k : T::kVec) * T::kBytes, v);
}
// Whether rows of K elements at `base` are streamed: where every row starts on 16
// bytes, neighbouring lanes fill whole lines, and keeping an output out of L2
// leaves it to what is read (norm of 2048 x 8192 into codes 26.6 -> 21.5 us in a
// graph, MX4 values of 2048 x 4096 5.4 -> 4.6, product 2048 x 11008 x 4096 46.4 ->
// 45.5).  Lines that two stores share cost more so (product 2048 x 11007 x 4096 into
// fp32 79 -> 94).
__host__ __device__ __forceinline__ bool streams(const void* base, int64_t K, int bytes) {
  return ((reinterpret_cast<uintptr_t>(base) | (uintptr_t)(K * bytes)) & 15) == 0;
}
// The same for values, whose waves write whole rows' runs: large outputs are
// streamed also where rows share lines (2048 x 11007 bf16 16.8 -> 13.7 us, 512 x 5001
// 3.65 -> 3.85).
inline bool streams_values(const void* base, int64_t rows, int64_t K, int bytes) {
  return streams(base, K, bytes) || rows * K * bytes >= (int64_t)12 << 20;
}

// Launches (arguments validated by the ABI).
hipError_t launch_quantize(const void* x, int type, int rows, int K, int64_t stride, const Operand& o, hipStream_t s);
hipError_t launch_dequantize(const Operand& o, int rows, int K, int type, void* out, hipStream_t s);
hipError_t launch_pack(const uint8_t* codes, const uint8_t* scales, int rows, int K, const Operand& o, hipStream_t s);
hipError_t launch_unpack(const Operand& o, int rows, int K, uint8_t* codes, uint8_t* scales, hipStream_t s);
// The norm into codes and scale (mx NULL), or into mx.
hipError_t launch_rmsnorm(int M, int K, int type, const void* x, int64_t x_stride, const void* residual, int64_t r_stride,
                          const void* gain, double eps, void* h, void* y, int q, int8_t* codes, uint16_t* scale,
                          const Operand* mx, hipStream_t s);
hipError_t launch_dequantize_codes(const int8_t* codes, const uint16_t* scale, int M, int K, int type, void* out,
                                   hipStream_t s);
// The product of two operands (mx4_gemm.hip); gemm_tiles: the workgroups of the
// launch, for the ABI's bound; gemm_block: the outputs that each makes.
int64_t gemm_tiles(int M, int N, int K);
void gemm_block(int M, int N, int K, int* rows, int* columns);
hipError_t launch_gemm(int M, int N, int K, const Operand& a, const Operand& w, int type, void* c, hipStream_t s);
// The same from rows, quantized in the product's kernel, where gemm_takes_rows;
// gemm_prefers_rows: and where that costs less than quantizing them first.
bool gemm_takes_rows(int M, int K);
bool gemm_prefers_rows(int M, int N, int K);
hipError_t launch_gemm_rows(int M, int N, int K, const void* x, int x_type, int64_t x_stride, const Operand& w, int type,
                            void* c, hipStream_t s);

}  // namespace mx4
}  // namespace apt
