// mx4_thin.h - the product of two MX4 operands for few rows of activations, or
// of weights, for gfx950.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 weight rows and 128 elements as 1 KB
// of the operand in lane order, and multiplies them with up to 16 activation rows.
// A workgroup owns 16 or 32 weight rows and up to 64 activation rows; its waves
// take the steps of K in turn, straight from memory into registers, and add their
// sums through LDS in the order of the waves.  So a workgroup has no barrier
// before its end and four times a tile's loads in flight for its outputs, and small
// ones fill the chip where tiles of 128 columns do not.
//
// What it reads bounds it.  One row: the weights, 1 x 11008 x 4096 5.8 us in a graph
// (a launch's 1.5 included), 24 MB at the rate of a large copy.  More rows: what a
// compute unit takes in, about 105 bytes a ns, 64 x 4096 x 11008 7.6 us in blocks of
// 32 x 32 (375 KB a unit), 8.8 in 64 x 16 (470 KB), 9.3 in 32 x 16.
//
// Activations of an operand come three steps ahead of their use where registers
// allow (one step ahead: 1 x 11008 x 4096 6.1 us, 32 x 11008 x 4096 7.2 instead of
// 6.8), from LDS one.
//
// The four scales of a lane's dword belong to blocks b, b + 2, b + 4, b + 6 of
// the step; lane group q = lane / 16 multiplies blocks q and q + 4, bytes
// q / 2 and q / 2 + 2 of half q mod 2, so the upper groups shift their dword by
// a byte and the MFMAs take bytes 0 and 2.
#pragma once

#include "mx4_tile.h"

namespace apt {
namespace mx4 {

// waves of a workgroup (1 x 11008 x 4096, activations a step ahead: 6.1 us, with 8
// waves 6.6 and with 16 9.4)
constexpr int kThinWaves = 4;

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
  int steps;
  Operand a, w;       // a: unused with rows
  uint8_t* c;
  // activations as rows (thin_kernel of an element type)
  const uint8_t* x;
  int64_t x_stride;   // elements
  int K;
};

__device__ __forceinline__ void store_output(uint8_t* c, int type, int64_t at, float v) {
  if (type == APT_TYPE_FP32) reinterpret_cast<float*>(c)[at] = v;
  else reinterpret_cast<uint16_t*>(c)[at] = type == APT_TYPE_FP16 ? Half::from_float(v) : Bf16::from_float(v);
}

// Rows quantized into LDS by a workgroup: the 16 bytes of block b of step t of
// row m at ((t * 8 + b) * M + m) * 16, behind them the scale dword of half h at
// ((t * 2 + h) * M + m) * 4.
inline size_t thin_lds_bytes(int M, int K) { return (size_t)steps(K) * M * (kStep / 2 + kStep / kBlock); }

// A thread's share of them: groups of eight elements, four neighbouring lanes to
// a block, kHeld at a time.  load() issues the first loads of a batch and
// store() converts it.
template <class X>
struct RowShare {
  static constexpr int kHeld = 2, kPieces = 8 / X::kVec;
  u32x4 v[kHeld][kPieces];

  // x / d, exact for the few thousand groups of eight here: x + 0.5 stays 0.5 / d
  // of the quotient away from an integer, the estimate of 1 / d 2^-22 of it.
  static __device__ __forceinline__ int quotient(int x, int d) {
    return (int)(((float)x + 0.5f) * __builtin_amdgcn_rcpf((float)d));
  }
  __device__ __forceinline__ void load(const ThinParams& p, int i0) {
    const int per_row = p.steps * (kStep / 8), all = per_row * p.M;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int x = min(i0 + i * kThinWaves * kWave, all - 1);
      const int m = quotient(x, per_row), k = (x - m * per_row) * 8;
      const uint8_t* const row = p.x + m * p.x_stride * X::kBytes;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = load_near<X>(row, k + j * X::kVec, p.K);
    }
  }
  __device__ __forceinline__ void store(const ThinParams& p, uint8_t* lds, int i0) {
    const int per_row = p.steps * (kStep / 8), all = per_row * p.M;
    uint8_t* const scales = lds + p.steps * p.M * (kStep / 2);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int x = i0 + i * kThinWaves * kWave;
      const int row = quotient(min(x, all - 1), per_row), y = min(x, all - 1) - row * per_row;  // eighth y of the row
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = settle<X>(v[i][j], y * 8 + j * X::kVec, p.K);
      uint32_t m = 0u;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) m = fold_magnitude<X>(m, v[i][j]);
      m = widest<X>(m);
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));  // lane ^ 1
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));  // lane ^ 2
      const uint32_t byte = scale_byte<X>(m);
      const uint32_t c = byte == 255u ? 0u : codes_of<X>(v[i], scale_of(byte));
      if (x >= all) continue;
      const int block = y / 4;
      *reinterpret_cast<uint32_t*>(lds + (block * p.M + row) * 16 + y % 4 * 4) = c;
      if (y % 4 == 0) scales[((block / 8 * 2 + block % 2) * p.M + row) * 4 + block % 8 / 2] = (uint8_t)byte;
    }
  }
};

// MT, NT: groups of 16 activation and weight rows of a workgroup.  KA, DA: steps of
// weights and of activations that a wave holds; KA is a multiple of DA.  X: void
// for an operand, or the element type of the rows that the workgroup quantizes
// into LDS itself (MT = 1).
template <int MT, int NT, int KA, int DA, class X>
__global__ __launch_bounds__(kThinWaves* kWave) void thin_kernel(ThinParams p) {
  constexpr int KW = kThinWaves;
  constexpr bool kRows = !std::is_void<X>::value;
  extern __shared__ __attribute__((aligned(16))) uint8_t rows_lds[];
  __shared__ float sums[KW][MT * NT * 256];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, q = lane / 16;
  const int S = p.steps;
  const unsigned across = ((unsigned)p.w.groups + NT - 1) / NT;
  const int64_t g0 = (int64_t)(blockIdx.x % across) * NT;  // first weight row group
  const int row0 = blockIdx.x / across * (MT * 16);        // first activation row
  const int shift = q / 2 * 8;

  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  u32x4 w[KA][NT][2], a[DA][MT][2];
  uint32_t sw[KA][NT], sa[DA][MT];
  // (groups and rows that are not there read the last one: their sums are not
  // stored; steps that are not there read the last one and are not multiplied)
  const uint8_t* wc[NT];
  const uint8_t* ws[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t g = min(g0 + j, p.w.groups - 1);
    wc[j] = p.w.codes + g * S * kCodeBytes + lane * 16;
    ws[j] = p.w.scales + g * S * kScaleBytes + q % 2 * 64 + s * 4;
  }
  auto load_w = [&](int u, int t) __attribute__((always_inline)) {
    const int64_t at = min(t, S - 1);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      w[u][j][0] = *reinterpret_cast<const u32x4*>(wc[j] + at * kCodeBytes);
      w[u][j][1] = *reinterpret_cast<const u32x4*>(wc[j] + at * kCodeBytes + 1024);
      sw[u][j] = *reinterpret_cast<const uint32_t*>(ws[j] + at * kScaleBytes);
    }
  };
  const uint8_t* ac[MT];
  const uint8_t* as[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = min(row0 + i * 16 + s, p.M - 1);
    if constexpr (kRows) {
      ac[i] = rows_lds + (q * p.M + m) * 16;
      as[i] = rows_lds + S * p.M * (kStep / 2) + (q % 2 * p.M + m) * 4;
    } else {
      ac[i] = p.a.codes + (int64_t)(m / 16) * S * kCodeBytes + q * 256 + m % 16 * 16;
      as[i] = p.a.scales + (int64_t)(m / 16) * S * kScaleBytes + q % 2 * 64 + m % 16 * 4;
    }
  }
  const int64_t a_step = kRows ? p.M * (kStep / 2) : kCodeBytes, as_step = kRows ? p.M * (kStep / kBlock) : kScaleBytes;
  const int a_half = kRows ? p.M * (kStep / 4) : 1024;
  auto load_a = [&](int u, int t) __attribute__((always_inline)) {
    const int64_t at = min(t, S - 1);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      a[u][i][0] = *reinterpret_cast<const u32x4*>(ac[i] + at * a_step);
      a[u][i][1] = *reinterpret_cast<const u32x4*>(ac[i] + at * a_step + a_half);
      sa[u][i] = *reinterpret_cast<const uint32_t*>(as[i] + at * as_step);
    }
  };
  if constexpr (kRows) {
    // the rows' loads leave before the weights', whose arrival then overlaps the
    // conversion (loads return in order)
    RowShare<X> share;
    share.load(p, threadIdx.x);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < KA; ++u) load_w(u, wave + u * KW);
    __builtin_amdgcn_sched_barrier(0);
    share.store(p, rows_lds, threadIdx.x);
    const int all = S * (kStep / 8) * p.M;
    for (int i = RowShare<X>::kHeld * KW * kWave; i < all; i += RowShare<X>::kHeld * KW * kWave) {
      share.load(p, i + threadIdx.x);
      share.store(p, rows_lds, i + threadIdx.x);
    }
    lds_barrier();
    load_a(0, wave);
  } else {
#pragma unroll
    for (int u = 0; u < KA; ++u) {
      if (u + 1 < DA) load_a(u, wave + u * KW);
      load_w(u, wave + u * KW);
    }
  }
  auto multiply = [&](int u) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int x = (int)(sw[u][j] >> shift);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int y = (int)(sa[u % DA][i] >> shift);
        acc[i][j] = mfma16(w[u][j][0], a[u % DA][i][0], acc[i][j], 0, x, y);
        acc[i][j] = mfma16(w[u][j][1], a[u % DA][i][1], acc[i][j], 1, x, y);
      }
    }
  };
  // while steps follow: each multiplied step's registers take the loads of the
  // step KA turns on
  int t0 = wave;
  for (; t0 + KW * KA < S; t0 += KW * KA) {
#pragma unroll
    for (int u = 0; u < KA; ++u) {
      const int t = t0 + u * KW;
      load_a((u + DA - 1) % DA, t + (DA - 1) * KW);
      __builtin_amdgcn_sched_barrier(0);
      multiply(u);
      load_w(u, t + KA * KW);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int u = 0; u < KA; ++u) {
    const int t = t0 + u * KW;
    if (u + DA - 1 < KA) load_a((u + DA - 1) % DA, t + (DA - 1) * KW);
    __builtin_amdgcn_sched_barrier(0);
    if (t < S) multiply(u);
  }
  // lane (s, q) holds weight rows 4 q + 0..3 of activation row s
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) *reinterpret_cast<v4f*>(&sums[wave][(i * NT + j) * 256 + s * 16 + q * 4]) = acc[i][j];
  lds_barrier();
  for (int x = threadIdx.x; x < MT * NT * 256; x += KW * kWave) {
    const int r = x / (NT * 16), c = x % (NT * 16);
    const int at = (r / 16 * NT + c / 16) * 256 + r % 16 * 16 + c % 16;
    const int64_t n = g0 * 16 + c;
    float v = sums[0][at];
#pragma unroll
    for (int k = 1; k < KW; ++k) v += sums[k][at];
    if (row0 + r < p.M && n < p.N) store_output(p.c, p.type, (row0 + r) * (int64_t)p.N + n, v);
  }
}

}  // namespace mx4
}  // namespace apt
