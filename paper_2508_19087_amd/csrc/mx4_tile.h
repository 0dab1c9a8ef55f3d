// mx4_tile.h - the tiled product of two MX4 operands for many rows, for gfx950.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies the codes as they lie in the
// operand: lane l gives row l mod 32 and block l / 32 of a K of 64 (16 bytes),
// and byte i of a dword gives its scale, so four MFMAs use up a step of 256 with
// one dword of scales per 32 rows.
//
// A workgroup of four waves makes MB * 32 rows by NB * 128 columns; each wave
// owns NB * 32 of the columns for all rows.  Its weights come straight from
// memory into registers (no other wave needs them), WD - 1 steps ahead (three for
// 128 columns, one for 256, whose sums take the registers); the activations,
// which all four waves need, go to LDS by direct loads, three steps ahead in a
// ring of four stages, and each fragment is read back two MFMA groups before its
// use.  One barrier per step, in its middle: it makes the next step's stage visible
// early enough that the first fragments and scales of that step are read before
// this one ends, and it frees the stage of the step before.
//
// 2048 x 11008 x 4096 (128 x 256 tiles, bf16 output) takes 46 to 47 us in a graph,
// 3.9 to 4.0 PFLOP/s, 16384 cubed 1755 to 1790 us or 4.9 to 5.0.  Clock stamps in
// the kernel: it runs at 1.50 to 1.55 GHz, with all units at dense products of
// random codes (16384 cubed: 1.37 to 1.42).  Its MFMAs alone, in the same two rounds
// of tiles, the second a third full, take 33 us at 1.6 to 1.7.  The rest is the
// epilogues, 3.9 us in each round, and waits for loads: a tile takes 39600 cycles,
// its MFMAs alone 27500.  Which tiles share their weights in the cache makes no
// difference.
// With about a tile per unit the ends count: the first step begins when its own
// loads have landed, not those of the three that follow (256 x 11008 x 4096 10.6
// us instead of 11.2, 333 x 5003 x 2999 7.3 instead of 7.6).
#pragma once

#include <type_traits>

#include "mx4.h"

namespace apt {
namespace mx4 {

constexpr int kWave = 64;
constexpr int kTileWaves = 4;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct GemmParams {
  int M, N;
  Operand a, w;
  uint8_t* c;
  int tiles_m, tiles_n;
};

__device__ __forceinline__ v8i operand_of(u32x4 v) {
  return v8i{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}
// The MFMA of 64 elements of K whose scales are byte i of the scale dwords.
__device__ __forceinline__ v16f mfma32(u32x4 w, u32x4 a, v16f c, int i, int sw, int sa) {
  switch (i) {
    case 0: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(w), operand_of(a), c, 4, 4, 0, sw, 0, sa);
    case 1: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(w), operand_of(a), c, 4, 4, 1, sw, 1, sa);
    case 2: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(w), operand_of(a), c, 4, 4, 2, sw, 2, sa);
    default: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand_of(w), operand_of(a), c, 4, 4, 3, sw, 3, sa);
  }
}

// Pins a value to this place of the program (kAcc: in an accumulation register).
template <bool kAcc>
__device__ __forceinline__ void keep(const v16f& x) {
  if constexpr (kAcc) asm volatile("" ::"a"(x));
  else asm volatile("" ::"v"(x));
}

// Four neighbouring outputs as bits of T: two dwords, or four of Float.
template <class T>
__device__ __forceinline__ u32x2 join4(float a, float b, float c, float d) {
  return u32x2{T::pair(a, b), T::pair(c, d)};
}

// WD: steps whose weights a wave holds, 2 or 4 (the loads run WD - 1 steps ahead).
template <class T, int MB, int NB, int WD>
__global__ __launch_bounds__(kTileWaves* kWave, (MB * NB >= 12 ? 1 : 2)) void tile_kernel(GemmParams p) {
  constexpr int kACodes = MB * 2 * kCodeBytes, kAScales = MB * 2 * kScaleBytes;
  constexpr int kSlot = 32 * (128 + 16);  // epilogue: 32 rows of 128 bytes or 16 of 256, padded
  constexpr int kStage = kACodes + kAScales > kSlot ? kACodes + kAScales : kSlot;
  constexpr int kSlots = 4 * MB;  // MFMA groups of a step
  __shared__ __attribute__((aligned(16))) uint8_t stage0[kStage];
  __shared__ __attribute__((aligned(16))) uint8_t stage1[kStage];
  __shared__ __attribute__((aligned(16))) uint8_t stage2[kStage];
  __shared__ __attribute__((aligned(16))) uint8_t stage3[kStage];

  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 32, h = lane / 32;
  const int S = p.a.steps;

  // Tile of this workgroup: workgroups are dealt round-robin to the 8 XCDs,
  // each of which takes a contiguous run of tiles in panels of 8 tile rows,
  // walked column by column, so that the tiles in flight on an XCD share both
  // operands in its L2.
  int m0, n0;
  {
    const int tiles = p.tiles_m * p.tiles_n;
    const int x = blockIdx.x % 8, i = blockIdx.x / 8;
    const int t = x * (tiles / 8) + min(x, tiles % 8) + i;
    const int panel = t / (8 * p.tiles_n), rest = t % (8 * p.tiles_n);
    const int ph = min(8, p.tiles_m - panel * 8);
    m0 = panel * 8 + rest % ph;
    n0 = rest / ph;
  }
  // first row groups of the tile, and the last of the operands (rows past the
  // edge read that one: their outputs are not stored)
  const int64_t ga0 = (int64_t)m0 * (MB * 2), gw0 = (int64_t)n0 * (NB * 8);
  const int ga_last = (int)min(p.a.groups - 1 - ga0, (int64_t)(MB * 2 - 1));
  const int gw_last = (int)min(p.w.groups - 1 - gw0, (int64_t)(NB * 8 - 1));
  auto resource = [](const uint8_t* base, int64_t first, int S, int bytes, int count) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base) + first * S * bytes, 0,
                                             (uint32_t)count * (uint32_t)S * (uint32_t)bytes, 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t ac = resource(p.a.codes, ga0, S, kCodeBytes, ga_last + 1);
  const __amdgpu_buffer_rsrc_t as = resource(p.a.scales, ga0, S, kScaleBytes, ga_last + 1);
  const __amdgpu_buffer_rsrc_t wc = resource(p.w.codes, gw0, S, kCodeBytes, gw_last + 1);
  const __amdgpu_buffer_rsrc_t ws = resource(p.w.scales, gw0, S, kScaleBytes, gw_last + 1);

  uint32_t w_off[NB], ws_off[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const uint32_t g = (uint32_t)min((wave * NB + b) * 2 + r / 16, gw_last) * (uint32_t)S;
    w_off[b] = g * kCodeBytes + h * 256 + r % 16 * 16;
    ws_off[b] = g * kScaleBytes + h * 64 + r % 16 * 4;
  }
  auto load_w = [&](int t, int b, int i) __attribute__((always_inline)) -> u32x4 {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wc, w_off[b] + i * 512, (uint32_t)t * kCodeBytes, 0));
  };
  auto load_ws = [&](int t, int b) __attribute__((always_inline)) -> int {
    return (int)__builtin_amdgcn_raw_buffer_load_b32(ws, ws_off[b], (uint32_t)t * kScaleBytes, 0);
  };
  // piece k of the wave's share of a step of A: 1 KB of codes, then 256 bytes
  // (two groups) of scales
  constexpr int kScalePieces = (MB + kTileWaves - 1) / kTileWaves;
  constexpr int kPieces = MB + kScalePieces;
  typedef __attribute__((address_space(3))) void* lds_t;
  auto load_a = [&](uint8_t* stage, int t, int k) __attribute__((always_inline)) {
    if (k < MB) {
      const int x = wave * MB + k;
      const uint32_t g = (uint32_t)min(x / 2, ga_last) * (uint32_t)S;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ac, (lds_t)(stage + x * 1024), 16, lane * 16,
                                               (g + (uint32_t)t) * kCodeBytes + x % 2 * 1024, 0, 0);
    } else {
      // (32-row block; where blocks do not go round, waves write the same bytes twice: no branch)
      const int x = min(wave + (k - MB) * kTileWaves, MB - 1);
      const uint32_t g = (uint32_t)min(x * 2 + lane / 32, ga_last) * (uint32_t)S;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(as, (lds_t)(stage + kACodes + x * 256), 4,
                                               g * kScaleBytes + lane % 32 * 4, (uint32_t)t * kScaleBytes, 0, 0);
    }
  };
  const int a_lane = r / 16 * kCodeBytes + h * 256 + r % 16 * 16;
  const int as_lane = kACodes + r / 16 * kScaleBytes + h * 64 + r % 16 * 4;
  // fragment of MFMA group s: rows s mod MB, 64 elements s / MB of the step
  auto read_a = [&](const uint8_t* stage, int s) __attribute__((always_inline)) -> u32x4 {
    return *reinterpret_cast<const u32x4*>(stage + a_lane + s % MB * (2 * kCodeBytes) + s / MB * 512);
  };
  auto read_as = [&](const uint8_t* stage, int a) __attribute__((always_inline)) -> int {
    return *reinterpret_cast<const int*>(stage + as_lane + a * (2 * kScaleBytes));
  };

  v16f acc[NB][MB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[b][a][v] = 0.0f;

  u32x4 w_[WD][NB][4], af[4];
  int sw_[WD][NB], sa_[2][MB];

  // Step t, the x-th of four: multiplies stage `cur`; reads the first fragments
  // of the next step from `nxt` and loads step t + 3 of A into `far` and the
  // weights of step t + WD - 1.
  // kLoads: the step loads; the steps behind the last whole four do not, all they
  // need being under way by then (but for the weights where WD = 2).
  auto step = [&](uint8_t* cur, uint8_t* nxt, uint8_t* far, int x, int t, auto kLoads) __attribute__((always_inline)) {
    u32x4(&w)[NB][4] = w_[x % WD];
    u32x4(&wn)[NB][4] = w_[(x + WD - 1) % WD];
    int(&sw)[NB] = sw_[x % WD];
    int(&swn)[NB] = sw_[(x + WD - 1) % WD];
    int(&sa)[MB] = sa_[x % 2];
    int(&san)[MB] = sa_[(x + 1) % 2];
    const int t1 = min(t + WD - 1, S - 1), t3 = min(t + 3, S - 1);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int i = s / MB, a = s % MB;
      if (s == kSlots / 2) {
        // Loads since those of step t + 1 of A, issued in step t - 2: a step's
        // share of A, a step of weights and (less than) half of one.  Steps that
        // do not load wait for everything: a count would hold loads that the
        // compiler leaves out where nothing reads them.
        constexpr int kSince = kLoads.value ? kPieces + 5 * NB + 2 * NB : 0;
        static_assert(kSince < 64, "vmcnt counts to 63");
        __builtin_amdgcn_s_waitcnt(0x0F70 | (kSince & 15) | (kSince >> 4) << 14);
        __builtin_amdgcn_s_barrier();
      }
      // the fragment two groups ahead, the next step's scales
      af[(s + 2) % 4] = s + 2 < kSlots ? read_a(cur, s + 2) : read_a(nxt, s + 2 - kSlots);
      if (s >= kSlots - MB) san[a] = read_as(nxt, a);
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][a] = mfma32(w[b][i], af[s % 4], acc[b][a], i, sw[b], sa[a]);
      // the weights' loads over the whole step, those of A over its second half
#pragma unroll
      for (int x = 0; x < 5 * NB; ++x)
        if ((kLoads.value || WD == 2) && x * kSlots / (5 * NB) == s) {
          if (x < NB) swn[x] = load_ws(t1, x);
          else wn[(x - NB) % NB][(x - NB) / NB] = load_w(t1, (x - NB) % NB, (x - NB) / NB);
        }
#pragma unroll
      for (int x = 0; x < kPieces; ++x)
        if (kLoads.value && kSlots / 2 + x * (kSlots / 2) / kPieces == s) load_a(far, t3, x);
      __builtin_amdgcn_sched_barrier(0);
    }
    // (an empty use of every accumulator: the step's MFMAs stay in it)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int a = 0; a < MB; ++a) keep<(MB * NB >= 12)>(acc[b][a]);
    __builtin_amdgcn_sched_barrier(0);
  };

  // The first loads, in the order of their use: step 0 begins when its own have
  // landed.  Where a wave holds two steps of weights, those of step 0 come behind
  // A of step 1, so that as many loads follow that as later (kSince).
  auto first_a = [&](uint8_t* stage, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < kPieces; ++x) load_a(stage, min(t, S - 1), x);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto first_w = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      sw_[t][b] = load_ws(min(t, S - 1), b);
#pragma unroll
      for (int i = 0; i < 4; ++i) w_[t][b][i] = load_w(min(t, S - 1), b, i);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  first_a(stage0, 0);
  if constexpr (WD == 4) first_w(0);
  first_a(stage1, 1);
  first_w(WD == 4 ? 1 : 0);
  first_a(stage2, 2);
  if constexpr (WD == 4) first_w(2);
  constexpr int kBehind = 2 * kPieces + (WD - 1) * 5 * NB;  // loads behind those of stage0
  static_assert(kBehind < 64, "vmcnt counts to 63");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (kBehind & 15) | (kBehind >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  af[0] = read_a(stage0, 0);
  af[1] = read_a(stage0, 1);
#pragma unroll
  for (int a = 0; a < MB; ++a) sa_[0][a] = read_as(stage0, a);
  __builtin_amdgcn_sched_barrier(0);
  int t = 0;
  for (; t + 3 < S; t += 4) {
    step(stage0, stage1, stage3, 0, t, std::true_type{});
    step(stage1, stage2, stage0, 1, t + 1, std::true_type{});
    step(stage2, stage3, stage1, 2, t + 2, std::true_type{});
    step(stage3, stage0, stage2, 3, t + 3, std::true_type{});
  }
  if (t < S) step(stage0, stage1, stage3, 0, t, std::false_type{});
  if (t + 1 < S) step(stage1, stage2, stage0, 1, t + 1, std::false_type{});
  if (t + 2 < S) step(stage2, stage3, stage1, 2, t + 2, std::false_type{});

  // ---- epilogue: through the wave's slot (stage `wave`), so that stores are whole
  // runs of all its columns of an output row (2048 x 11007 x 4096 into fp32, whose
  // rows share lines: 75 to 77 us with runs of 256 bytes, 79 with two of 128; 2048 x
  // 11008 x 4096, whose rows do not, 52).  The MFMA
  // leaves lane (r, h) columns 8 g + 4 h + 0..3 of row r.
  __builtin_amdgcn_s_waitcnt(0x0070);  // the last (unused) loads have landed
  __builtin_amdgcn_s_barrier();
  // A pass takes 32 rows of 64 or 128 bytes, or 16 of 256.
  constexpr int kRowBytes = NB * 32 * T::kBytes, kPassRows = kRowBytes > 128 ? 16 : 32;
  constexpr int kStride = kRowBytes + 16;
  static_assert(kPassRows * kStride <= kSlot, "a pass fits its slot");
  uint8_t* const slot = wave == 0 ? stage0 : wave == 1 ? stage1 : wave == 2 ? stage2 : stage3;
  const int nw = n0 * (NB * 128) + wave * (NB * 32);
  constexpr int kRowPieces = kRowBytes / 16;  // 16-byte pieces of a row
  constexpr int kRowsAtOnce = kWave / kRowPieces;
  auto epilogue = [&](auto kStream) __attribute__((always_inline)) {
    if (nw >= p.N) return;  // uniform: no output here
#pragma unroll
    for (int a = 0; a < MB; ++a) {
#pragma unroll
      for (int r0 = 0; r0 < 32; r0 += kPassRows) {
        if ((int64_t)m0 * (MB * 32) + a * 32 + r0 >= p.M) continue;
        if (kPassRows == 32 || r / kPassRows * kPassRows == r0) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              uint8_t* const at = slot + (r - r0) * kStride + (b * 32 + g * 8 + h * 4) * T::kBytes;
              const v16f& c = acc[b][a];
              if constexpr (T::kBytes == 4)
                *reinterpret_cast<v4f*>(at) = v4f{c[g * 4], c[g * 4 + 1], c[g * 4 + 2], c[g * 4 + 3]};
              else
                *reinterpret_cast<u32x2*>(at) = join4<T>(c[g * 4], c[g * 4 + 1], c[g * 4 + 2], c[g * 4 + 3]);
            }
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);  // this wave's LDS writes are done
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < kPassRows / kRowsAtOnce; ++j) {
          const int row = j * kRowsAtOnce + lane / kRowPieces, piece = lane % kRowPieces;
          const u32x4 v = *reinterpret_cast<const u32x4*>(slot + row * kStride + piece * 16);
          const int64_t m = (int64_t)m0 * (MB * 32) + a * 32 + r0 + row;
          const int n = nw + piece * T::kVec;
          if (m < p.M) store_vector<T, kStream.value>(p.c + m * p.N * T::kBytes, n, p.N, v);
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);  // reads done before the slot is rewritten
        __builtin_amdgcn_wave_barrier();
      }
    }
  };
  if (streams(p.c, p.N, T::kBytes)) epilogue(std::true_type{});
  else epilogue(std::false_type{});
}

}  // namespace mx4
}  // namespace apt
