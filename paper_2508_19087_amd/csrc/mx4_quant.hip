// mx4_quant.hip - rows to MX4 operands and back, for gfx950.
//
// All of it is bound by memory: quantizing reads 2 or 4 bytes per element and
// writes 17/32; the arithmetic (a maximum over integer bits, and one scaled
// conversion instruction per two elements, which rounds to nearest even and
// saturates) hides behind the loads.
//
// A wave quantizes eight rows of one step (256 elements) of K: eight lanes to a
// row, four to a block, eight elements to a lane.  A load instruction then reads
// whole lines, two blocks of each row, a block's largest magnitude takes two lane
// swaps, and the codes leave in runs of 128 bytes; a lane sees its block of all
// four instructions, whose scales are one dword of the operand.  (With whole
// blocks to a lane, a wave took 16 rows and each load touched 64 lines: 64 x 4096
// fp16 3.4 us in a graph instead of 2.7, 2048 x 11008 bf16 11.1 instead of 10.1 and
// fp32 23.7 instead of 17.8, which are 57 and 102 MB.)  Values take four rows of
// a step per wave: 2048 x 11008 bf16 9.9 us and fp32 16.6 (16 rows: 10.3 and 17.3;
// 64 x 4096 2.55 and 2.78 instead of 3.3 and 4.1).
#include "mx4.h"

namespace apt {
namespace {

using namespace mx4;

constexpr int kWave = 64;
constexpr int kWaves = 4;
constexpr int kQuantizeParts = 2, kValueParts = 4;  // waves to 16 rows of a step

// (a struct: each argument of a launch takes its share of the host's time)
struct Rows {
  uint8_t* x;
  int rows, K;
  int64_t stride;  // elements
  Operand o;
};

template <class T>
__global__ __launch_bounds__(kWave* kWaves) void quantize_kernel(Rows a) {
  const uint8_t* const x = a.x;
  const int rows = a.rows, K = a.K;
  const int64_t stride = a.stride;
  const Operand o = a.o;
  constexpr int kPieces = 8 / T::kVec;  // vectors of a lane's eight elements
  const int lane = threadIdx.x % kWave;
  const int64_t at = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
  const int64_t unit = at / kQuantizeParts;
  if (unit >= o.groups * o.steps) return;
  const int64_t g = unit / o.steps;
  const int first = (int)(at % kQuantizeParts) * (kGroup / kQuantizeParts);
  if (g * kGroup + first >= rows) return;
  const int s = first + lane / 8, h = lane / 4 % 2, e = lane % 4;
  const int64_t row = g * kGroup + s;
  const bool real = row < rows;
  // (rows past the edge read the first row and store nothing)
  const uint8_t* const src = x + (real ? row : 0) * stride * T::kBytes;
  const int k0 = (int)(unit % o.steps) * kStep;
  u32x4 v[4][kPieces];
  auto place = [&](int i, int j) __attribute__((always_inline)) { return k0 + i * 2 * kBlock + lane % 8 * 8 + j * T::kVec; };
  if (k0 + kStep <= K) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = load_whole<T>(src, place(i, j));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = load_near<T>(src, place(i, j), K);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = settle<T>(v[i][j], place(i, j), K);
  }
  uint32_t bytes = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t m = 0u;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) m = fold_magnitude<T>(m, v[i][j]);
    m = widest<T>(m);
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));  // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));  // lane ^ 2
    const uint32_t byte = scale_byte<T>(m);
    const uint32_t c = byte == 255u ? 0u : codes_of<T>(v[i], scale_of(byte));
    if (real) *reinterpret_cast<uint32_t*>(o.codes + (unit * 8 + 2 * i + h) * 256 + s * 16 + e * 4) = c;
    bytes |= byte << (8 * i);
  }
  if (real && e == 0) *reinterpret_cast<uint32_t*>(o.scales + unit * kScaleBytes + h * 64 + s * 4) = bytes;
}

// A vector of values: of eight codes in 16-bit types, of four in fp32.
template <class T>
__device__ __forceinline__ u32x4 packed_values(uint32_t c, float scale, bool nan) {
  u32x4 v;
  if constexpr (T::kBytes == 4) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
    const float f[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = nan ? 0x7FC00000u : __builtin_bit_cast(uint32_t, f[j]);
    return v;
  } else if constexpr (T::kInf == Half::kInf) {
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, scale, 3));
  } else {
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = nan ? (T::kInf | 0x40u) * 0x00010001u : v[j];
  return v;
}

// Values of an operand.  A wave takes four rows of a step; its lanes take the
// elements of a row in order, eight at a time for 16-bit types (two rows at once)
// and four for fp32, so that every store instruction writes whole 512-byte or
// 1 KB runs.
template <class T, bool kStream>
__global__ __launch_bounds__(kWave* kWaves) void dequantize_kernel(Rows a) {
  uint8_t* const out = a.x;
  const int rows = a.rows, K = a.K;
  const Operand o = a.o;
  constexpr int kElems = T::kVec;                  // per lane and row
  constexpr int kAtOnce = kWave * kElems / kStep;  // rows per store
  constexpr int kTurns = kGroup / kAtOnce / kValueParts;
  const int lane = threadIdx.x % kWave;
  const int64_t at = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
  const int64_t unit = at / kValueParts;
  if (unit >= o.groups * o.steps) return;
  const int64_t g = unit / o.steps;
  const int first = (int)(at % kValueParts) * (kAtOnce * kTurns) + lane / (kStep / kElems);
  const int in_step = lane % (kStep / kElems) * kElems, b = in_step / kBlock;
  const int k = (int)(unit % o.steps) * kStep + in_step;
  uint32_t c[kTurns], e[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int s = first + kAtOnce * i;
    const uint8_t* const from = o.codes + (unit * 8 + b) * 256 + s * 16 + in_step % kBlock / 2;
    c[i] = kElems == 8 ? *reinterpret_cast<const uint32_t*>(from) : (uint32_t)*reinterpret_cast<const uint16_t*>(from);
    e[i] = o.scales[unit * kScaleBytes + b % 2 * 64 + s * 4 + b / 2];
  }
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int64_t row = g * kGroup + first + kAtOnce * i;
    if (row < rows)
      store_vector<T, kStream>(out + row * K * T::kBytes, k, K, packed_values<T>(c[i], scale_of(e[i]), e[i] == 255u));
  }
}

// Row-major codes and scale bytes into the operand (or back), a thread per
// block: once per model, so nothing of it is tuned (11008 x 4096, 24 MB in and out:
// 49 us, and back 47, where a large copy takes 9).
__global__ __launch_bounds__(256) void pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                   int rows, int K, Operand o) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t unit = i / 128;
  if (unit >= o.groups * o.steps) return;
  const int s = i % 16, b = (int)(i / 16 % 8);
  const int64_t row = unit / o.steps * kGroup + s;
  if (row >= rows) return;
  const int k = (int)(unit % o.steps) * kStep + b * kBlock;
  const int64_t row_bytes = ((int64_t)K + 1) / 2, blocks = ((int64_t)K + kBlock - 1) / kBlock;
  u32x4 c = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (k + 2 * j < K) {
      const uint32_t v = codes[row * row_bytes + k / 2 + j];
      c[j / 4] |= (k + 2 * j + 1 < K ? v : v & 15u) << (8 * (j % 4));
    }
  *reinterpret_cast<u32x4*>(o.codes + (unit * 8 + b) * 256 + s * 16) = c;
  o.scales[unit * kScaleBytes + b % 2 * 64 + s * 4 + b / 2] = k < K ? scales[row * blocks + k / kBlock] : 0;
}

__global__ __launch_bounds__(256) void unpack_kernel(Operand o, int rows, int K, uint8_t* __restrict__ codes,
                                                     uint8_t* __restrict__ scales) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t unit = i / 128;
  if (unit >= o.groups * o.steps) return;
  const int s = i % 16, b = (int)(i / 16 % 8);
  const int64_t row = unit / o.steps * kGroup + s;
  const int k = (int)(unit % o.steps) * kStep + b * kBlock;
  if (row >= rows || k >= K) return;
  const int64_t row_bytes = ((int64_t)K + 1) / 2, blocks = ((int64_t)K + kBlock - 1) / kBlock;
  const u32x4 c = *reinterpret_cast<const u32x4*>(o.codes + (unit * 8 + b) * 256 + s * 16);
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (k + 2 * j < K) codes[row * row_bytes + k / 2 + j] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
  scales[row * blocks + k / kBlock] = o.scales[unit * kScaleBytes + b % 2 * 64 + s * 4 + b / 2];
}

unsigned unit_blocks(const Operand& o, int parts) { return (unsigned)((o.groups * o.steps * parts + kWaves - 1) / kWaves); }

}  // namespace

namespace mx4 {

hipError_t launch_quantize(const void* x, int type, int rows, int K, int64_t stride, const Operand& o, hipStream_t s) {
  const dim3 grid(unit_blocks(o, kQuantizeParts)), block(kWave * kWaves);
  const Rows a{static_cast<uint8_t*>(const_cast<void*>(x)), rows, K, stride, o};  // (not written)
  switch (type) {
    case APT_TYPE_FP16: return launch_kernel(quantize_kernel<Half>, grid, block, 0, s, a);
    case APT_TYPE_BF16: return launch_kernel(quantize_kernel<Bf16>, grid, block, 0, s, a);
    default: return launch_kernel(quantize_kernel<Float>, grid, block, 0, s, a);
  }
}

template <class T>
static hipError_t launch_dequantize_of(const Operand& o, int rows, int K, void* out, hipStream_t s) {
  return launch_kernel(streams_values(out, rows, K, T::kBytes) ? dequantize_kernel<T, true> : dequantize_kernel<T, false>,
                       dim3(unit_blocks(o, kValueParts)), dim3(kWave * kWaves), 0, s, Rows{static_cast<uint8_t*>(out), rows, K, K, o});
}

hipError_t launch_dequantize(const Operand& o, int rows, int K, int type, void* out, hipStream_t s) {
  switch (type) {
    case APT_TYPE_FP16: return launch_dequantize_of<Half>(o, rows, K, out, s);
    case APT_TYPE_BF16: return launch_dequantize_of<Bf16>(o, rows, K, out, s);
    default: return launch_dequantize_of<Float>(o, rows, K, out, s);
  }
}

hipError_t launch_pack(const uint8_t* codes, const uint8_t* scales, int rows, int K, const Operand& o, hipStream_t s) {
  const dim3 grid((unsigned)((o.groups * o.steps + 1) / 2)), block(256);
  return launch_kernel(pack_kernel, grid, block, 0, s, codes, scales, rows, K, o);
}

hipError_t launch_unpack(const Operand& o, int rows, int K, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const dim3 grid((unsigned)((o.groups * o.steps + 1) / 2)), block(256);
  return launch_kernel(unpack_kernel, grid, block, 0, s, o, rows, K, codes, scales);
}

}  // namespace mx4
}  // namespace apt
