// mx4_gemm.hip - C = A * W^T of two MX4 operands on the block-scaled MFMA, for
// gfx950.
#include "mx4.h"

namespace apt {
namespace {

using namespace mx4;

constexpr int kWave = 64;
constexpr int kWaves = 4;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct GemmParams {
  int M, N;
  Operand a, w;
  uint8_t* c;
  int tiles_n;  // of 128 columns
};

template <class T>
__device__ __forceinline__ void store_value(uint8_t* c, int64_t at, float v) {
  if constexpr (T::kBytes == 4) reinterpret_cast<float*>(c)[at] = v;
  else reinterpret_cast<uint16_t*>(c)[at] = T::from_float(v);
}

__device__ __forceinline__ v8i operand_of(u32x4 v) {
  return v8i{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}

// 32 rows x 128 columns per workgroup, 32 x 32 per wave.
template <class T>
__global__ __launch_bounds__(kWave* kWaves) void gemm_kernel(GemmParams p) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int r = lane % 32, h = lane / 32;
  const int64_t m0 = (int64_t)(blockIdx.x / (unsigned)p.tiles_n) * 32;
  const int64_t n0 = (int64_t)(blockIdx.x % (unsigned)p.tiles_n) * 128 + wave * 32;
  if (n0 >= p.N) return;
  const int S = p.a.steps;
  // (rows past the edge read the last group: their outputs are not stored)
  const int64_t ga = min(m0 / 16 + r / 16, p.a.groups - 1), gw = min(n0 / 16 + r / 16, p.w.groups - 1);
  const uint8_t* const ac = p.a.codes + ga * S * kCodeBytes + h * 256 + r % 16 * 16;
  const uint8_t* const wc = p.w.codes + gw * S * kCodeBytes + h * 256 + r % 16 * 16;
  const uint8_t* const as = p.a.scales + ga * S * kScaleBytes + h * 64 + r % 16 * 4;
  const uint8_t* const ws = p.w.scales + gw * S * kScaleBytes + h * 64 + r % 16 * 4;
  v16f acc = {};
  for (int t = 0; t < S; ++t) {
    const int sa = *reinterpret_cast<const int*>(as + (int64_t)t * kScaleBytes);
    const int sw = *reinterpret_cast<const int*>(ws + (int64_t)t * kScaleBytes);
    u32x4 av[4], wv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      av[i] = *reinterpret_cast<const u32x4*>(ac + (int64_t)t * kCodeBytes + i * 512);
      wv[i] = *reinterpret_cast<const u32x4*>(wc + (int64_t)t * kCodeBytes + i * 512);
    }
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(wv[0]), operand_of(av[0]), acc, 4, 4, 0, sw, 0, sa);
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(wv[1]), operand_of(av[1]), acc, 4, 4, 1, sw, 1, sa);
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(wv[2]), operand_of(av[2]), acc, 4, 4, 2, sw, 2, sa);
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(wv[3]), operand_of(av[3]), acc, 4, 4, 3, sw, 3, sa);
  }
  const int64_t m = m0 + r;
  if (m >= p.M) return;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int64_t n = n0 + v / 4 * 8 + h * 4 + v % 4;
    if (n < p.N) store_value<T>(p.c, m * p.N + n, acc[v]);
  }
}

}  // namespace

namespace mx4 {

int64_t gemm_tiles(int M, int N, int K) {
  (void)K;
  return ((int64_t)M + 31) / 32 * (((int64_t)N + 127) / 128);
}

size_t gemm_workspace(int M, int N, int K) {
  (void)M, (void)N, (void)K;
  return 0;
}

hipError_t launch_gemm(int M, int N, int K, const Operand& a, const Operand& w, int type, void* c, void* workspace,
                       hipStream_t s) {
  (void)workspace;
  GemmParams p{M, N, a, w, static_cast<uint8_t*>(c), (int)(((int64_t)N + 127) / 128)};
  const dim3 grid((unsigned)gemm_tiles(M, N, K)), block(kWave * kWaves);
  switch (type) {
    case APT_TYPE_FP16: return launch_kernel(gemm_kernel<Half>, grid, block, 0, s, p);
    case APT_TYPE_BF16: return launch_kernel(gemm_kernel<Bf16>, grid, block, 0, s, p);
    default: return launch_kernel(gemm_kernel<Float>, grid, block, 0, s, p);
  }
}

}  // namespace mx4
}  // namespace apt
