// mx4_thin.h - the product of two MX4 operands for few rows of activations, for
// gfx950.
//
// With up to 64 rows the weights are the traffic, and the kernel is a stream of
// them: v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 weight rows and 128 elements
// as 1 KB of the operand in lane order, and multiplies them with up to 16
// activation rows.  A workgroup owns 16 weight rows; its waves take the steps of
// K in turn, each issuing the loads of kAhead steps before it multiplies, and
// add their sums through LDS in the order of the waves.
//
// The four scales of a lane's dword belong to blocks b, b + 2, b + 4, b + 6 of
// the step; lane group q = lane / 16 multiplies blocks q and q + 4, bytes
// q / 2 and q / 2 + 2 of half q mod 2, so the upper groups shift their dword by
// a byte and the MFMAs take bytes 0 and 2.
#pragma once

#include "mx4_tile.h"

namespace apt {
namespace mx4 {

constexpr int kThinRows = 64;  // activation rows, at most
constexpr int kThinWaves = 4;  // waves of a workgroup (8 and 16 are slower, as 1 x 11008 x 4096: 6.0, 6.6, 9.4 us)
constexpr int kAhead = 4;      // steps whose loads are in flight per wave

// The MFMA of half j of a step.
__device__ __forceinline__ v4f mfma16(u32x4 w, u32x4 a, v4f c, int j, int sw, int sa) {
  return j == 0 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand_of(w), operand_of(a), c, 4, 4, 0, sw, 0, sa)
                : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand_of(w), operand_of(a), c, 4, 4, 2, sw, 2, sa);
}

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

struct ThinParams {
  int M, N, type;
  Operand a, w;
  uint8_t* c;
};

__device__ __forceinline__ void store_output(uint8_t* c, int type, int64_t at, float v) {
  if (type == APT_TYPE_FP32) reinterpret_cast<float*>(c)[at] = v;
  else reinterpret_cast<uint16_t*>(c)[at] = type == APT_TYPE_FP16 ? Half::from_float(v) : Bf16::from_float(v);
}

// MT: groups of 16 activation rows.
template <int MT>
__global__ __launch_bounds__(kThinWaves* kWave) void thin_kernel(ThinParams p) {
  constexpr int KW = kThinWaves;
  __shared__ float sums[KW][MT * 256];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, q = lane / 16;
  const int S = p.a.steps;
  const int64_t g = blockIdx.x;  // weight row group
  const uint8_t* const wc = p.w.codes + g * S * kCodeBytes + lane * 16;
  const uint8_t* const ws = p.w.scales + g * S * kScaleBytes + q % 2 * 64 + s * 4;
  const int shift = q / 2 * 8;

  // (rows that are not there read the last one: their sums are not stored)
  const uint8_t* ac[MT];
  const uint8_t* as[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = min(i * 16 + s, p.M - 1);
    ac[i] = p.a.codes + (int64_t)(m / 16) * S * kCodeBytes + q * 256 + m % 16 * 16;
    as[i] = p.a.scales + (int64_t)(m / 16) * S * kScaleBytes + q % 2 * 64 + m % 16 * 4;
  }

  v4f acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  u32x4 w[kAhead][2], a[2][MT][2];
  uint32_t sw[kAhead], sa[2][MT];
  // (steps that are not there read the last one and are not multiplied)
  auto load_w = [&](int u, int t) __attribute__((always_inline)) {
    const int64_t at = min(t, S - 1);
    w[u][0] = *reinterpret_cast<const u32x4*>(wc + at * kCodeBytes);
    w[u][1] = *reinterpret_cast<const u32x4*>(wc + at * kCodeBytes + 1024);
    sw[u] = *reinterpret_cast<const uint32_t*>(ws + at * kScaleBytes);
  };
  auto load_a = [&](int u, int t) __attribute__((always_inline)) {
    const int64_t at = min(t, S - 1);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      a[u][i][0] = *reinterpret_cast<const u32x4*>(ac[i] + at * kCodeBytes);
      a[u][i][1] = *reinterpret_cast<const u32x4*>(ac[i] + at * kCodeBytes + 1024);
      sa[u][i] = *reinterpret_cast<const uint32_t*>(as[i] + at * kScaleBytes);
    }
  };
  load_a(0, wave);
#pragma unroll
  for (int u = 0; u < kAhead; ++u) load_w(u, wave + u * KW);
  auto multiply = [&](int u) __attribute__((always_inline)) {
    const int x = (int)(sw[u] >> shift);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int y = (int)(sa[u % 2][i] >> shift);
      acc[i] = mfma16(w[u][0], a[u % 2][i][0], acc[i], 0, x, y);
      acc[i] = mfma16(w[u][1], a[u % 2][i][1], acc[i], 1, x, y);
    }
  };
  // while steps follow: each multiplied step's registers take the loads of the
  // step kAhead turns on
  int t0 = wave;
  for (; t0 + KW * kAhead < S; t0 += KW * kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = t0 + u * KW;
      load_a((u + 1) % 2, t + KW);
      __builtin_amdgcn_sched_barrier(0);
      multiply(u);
      load_w(u, t + kAhead * KW);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int t = t0 + u * KW;
    if (u + 1 < kAhead) load_a((u + 1) % 2, t + KW);
    __builtin_amdgcn_sched_barrier(0);
    if (t < S) multiply(u);
  }
  // lane (s, q) holds weight rows 4 q + 0..3 of activation row s
#pragma unroll
  for (int i = 0; i < MT; ++i) *reinterpret_cast<v4f*>(&sums[wave][i * 256 + s * 16 + q * 4]) = acc[i];
  lds_barrier();
  for (int x = threadIdx.x; x < MT * 256; x += KW * kWave) {
    const int m = x / 16;
    const int64_t n = g * 16 + x % 16;
    float v = sums[0][x];
#pragma unroll
    for (int k = 1; k < KW; ++k) v += sums[k][x];
    if (m < p.M && n < p.N) store_output(p.c, p.type, m * (int64_t)p.N + n, v);
  }
}

}  // namespace mx4
}  // namespace apt
