// rmsnorm.hip - RMS norm of rows with the residual's addition in front and the
// operand of a quantized product behind (q-bit codes with a scale per row, or
// MX4), for gfx950.
//
// Bound by memory: 2 bytes per element of x and residual in, 2 of h and 1 (or
// 17/32) of the operand out.  A row is one workgroup's and stays in registers
// between its passes (sum of squares, largest magnitude of y, codes), each
// thread holding NV vectors of 8 elements; rows longer than the registers
// reach (NV = 0) are read again in each pass.  In a graph 2048 x 4096 into codes
// takes 13.0 us (59 MB, 4.5 TB/s; a large copy 5.1 to 5.2), into MX4 11.9, 1 x 4096
// 3.2 and 3.0: a launch and one trip to memory.  Traced among other kernels 13.7 and
// 12.3.
//
// The sum of squares runs in fp64.  A quantizer is a step function, and a y
// that moved by one rounding with the order of its row's sum would now and then
// move a code; squares of 11-bit values and their sums are exact to 2^-53 here,
// so the order all but never shows in f; y and its codes follow from f by single
// IEEE operations.
#include "mx4.h"
#include "rowcode.h"

namespace apt {
namespace {

using namespace mx4;

constexpr int kWave = 64;
constexpr int kMaxWaves = 16;

struct NormArgs {
  int M, K;
  const uint8_t* x;
  int64_t x_stride;  // elements
  const uint8_t* residual;
  int64_t r_stride;
  const uint8_t* gain;
  double inv_k, eps;  // 1 / K
  uint8_t* h;
  uint8_t* y;
  int q;
  int8_t* codes;
  uint16_t* scale;
  Operand mx;
};

// Eight elements of fp32 from a vector of 16-bit ones, and back.
template <class T>
__device__ __forceinline__ void spread(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = T::to_float((uint16_t)(v[i / 2] >> (16 * (i % 2))));
}
template <class T>
__device__ __forceinline__ u32x4 join(const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = T::pair(f[2 * i], f[2 * i + 1]);
  return v;
}

// Sum and largest value over the workgroup; `lds` holds a value per wave.  Within
// a wave four DPP steps give every 16-lane row its result and lane reads the
// wave's (through LDS, six dependent swaps of a double take about 0.4 us more).
template <int kCtrl>
__device__ __forceinline__ double add_dpp(double v) {
  const u32x2 b = __builtin_bit_cast(u32x2, v);
  const u32x2 o = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)b[0], kCtrl, 0xF, 0xF, false),
                   (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b[1], kCtrl, 0xF, 0xF, false)};
  return v + __builtin_bit_cast(double, o);
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  const u32x2 b = __builtin_bit_cast(u32x2, v);
  const u32x2 o = {(uint32_t)__builtin_amdgcn_readlane((int)b[0], lane), (uint32_t)__builtin_amdgcn_readlane((int)b[1], lane)};
  return __builtin_bit_cast(double, o);
}
__device__ __forceinline__ double block_sum(double v, double* lds) {
  v = add_dpp<0xB1>(v);   // lane ^ 1
  v = add_dpp<0x4E>(v);   // lane ^ 2
  v = add_dpp<0x141>(v);  // the row's half mirrored
  v = add_dpp<0x140>(v);  // the row mirrored
  v = (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
  const int waves = (int)blockDim.x / kWave;
  if (waves == 1) return v;
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  double sum = 0.0;
  for (int w = 0; w < waves; ++w) sum += lds[w];
  return sum;
}
// The same over kLanes neighbouring lanes (16, 32, or 64: a wave).
template <int kLanes>
__device__ __forceinline__ double lanes_sum(double v) {
  v = add_dpp<0xB1>(v);
  v = add_dpp<0x4E>(v);
  v = add_dpp<0x141>(v);
  v = add_dpp<0x140>(v);
  if (kLanes == 32) v += __shfl_xor(v, 16);
  if (kLanes == 64) v = (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
  return v;
}
template <int kLanes>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  if (kLanes == 64) return rowcode::wave_max(v);
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* lds) {
  v = rowcode::wave_max(v);
  const int waves = (int)blockDim.x / kWave;
  if (waves == 1) return v;
  if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  uint32_t m = 0u;
  for (int w = 0; w < waves; ++w) m = max(m, lds[w]);
  return m;
}

// 1 / sqrt(v), to 2^-50 or better (v a normal number, 0 or infinite): the
// hardware's estimate r, and with e = 1 - v r^2 the expansion of r (1 - e)^(-1/2)
// to second order, twice (an estimate good to 2^-14 suffices).
__device__ __forceinline__ double inverse_root(double v) {
  double r = __builtin_amdgcn_rsq(v);
  if (!(v > 0.0) || r == 0.0) return r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const double e = __builtin_fma(-v * r, r, 1.0);
    r = __builtin_fma(r * e, __builtin_fma(e, 0.375, 0.5), r);
  }
  return r;
}

// A row's codes from its largest magnitude: floor(h) of h = y / (2 s).  y and s
// have at most 11 significant bits, so an h that is no integer lies 2^-18 of
// itself or more away from one, while the product with the reciprocal is off by
// 2^-22 at most: lifted by |h| 2^-20 it passes the border of an integer and no
// other.  With a normal s, |h| is at most (2^q - 1) / 2 (1 + 2^-11) and its floor
// in range; a subnormal s may be far from the quotient it rounds, and h further
// out.
struct CodeScale {
  float rh;       // 0.5 / s
  uint32_t bits;  // s
  bool bad, clamp;
  template <class T>
  __device__ __forceinline__ void set(uint32_t m, int q) {
    const float top = (float)((1 << q) - 1);
    const _Float16 s16 = (_Float16)__fdiv_rn(T::to_float((uint16_t)m), top);
    bits = __builtin_bit_cast(uint16_t, s16);
    bad = m >= T::kInf || bits >= 0x7C00u;
    clamp = bits < 0x0400u;
    rh = !bad && bits != 0u ? 0.5f * __builtin_amdgcn_rcpf((float)s16) : 0.0f;
    if (bad) bits = 0x7E00u;
  }
  // codes of eight values, a byte each
  __device__ __forceinline__ u32x2 codes(const float (&y)[8], int q) const {
    if (bad) return u32x2{0u, 0u};
    int v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float h = y[i] * rh;
      asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(v[i]) : "v"(__builtin_fmaf(__builtin_fabsf(h), 0x1p-20f, h)));
    }
    if (clamp) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = min(max(v[i], -(1 << (q - 1))), (1 << (q - 1)) - 1);
    }
    u32x2 c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int* const b = v + 4 * i;
      c[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm((uint32_t)b[3], (uint32_t)b[2], 0x0C0C0400u),
                                   __builtin_amdgcn_perm((uint32_t)b[1], (uint32_t)b[0], 0x0C0C0400u), 0x05040100u);
    }
    return c;
  }
};

// T: element type; NV: vectors of 8 elements held per thread (0: none, the row
// is read again in each pass); LANES: 0, or the lanes that a row takes, several
// rows to a workgroup; kCodes: q-bit codes, else MX4; kWhole: K is a
// multiple of 8, so that no vector is cut by the row's end, and every row starts
// at a multiple of 16 bytes where it is written.
template <class T, int NV, int LANES, bool kCodes, bool kWhole>
__global__ __launch_bounds__(kWave* kMaxWaves) void rmsnorm_kernel(NormArgs a) {
  __shared__ double lds_sum[kMaxWaves];
  __shared__ uint32_t lds_max[kMaxWaves];
  const int K = a.K;
  const int tid = LANES ? threadIdx.x % LANES : threadIdx.x;
  const int threads = LANES ? LANES : (int)blockDim.x;  // of the row
  // MX4: the 16 rows of a group share the operand's lines, and workgroups are
  // dealt round-robin to the 8 XCDs: group g's rows go to XCD g mod 8
  const int64_t row = LANES ? (int64_t)blockIdx.x * (blockDim.x / LANES) + threadIdx.x / LANES
                    : kCodes ? (int64_t)blockIdx.x
                             : (int64_t)(blockIdx.x / 128) * 128 + blockIdx.x % 8 * 16 + blockIdx.x / 8 % 16;
  if (row >= a.M) return;
  auto row_sum = [&](double v) __attribute__((always_inline)) {
    if constexpr (LANES > 0) return lanes_sum<LANES>(v);
    else return block_sum(v, lds_sum);
  };
  auto row_max = [&](uint32_t v) __attribute__((always_inline)) {
    if constexpr (LANES > 0) return lanes_max<LANES>(v);
    else return block_max(v, lds_max);
  };
  const uint8_t* const x = a.x + row * a.x_stride * 2;
  const uint8_t* const r = a.residual != nullptr ? a.residual + row * a.r_stride * 2 : nullptr;
  uint8_t* const hrow = a.h != nullptr ? a.h + row * K * 2 : nullptr;
  uint8_t* const yrow = a.y != nullptr ? a.y + row * K * 2 : nullptr;
  // elements that are written: MX4 rows end on a step
  const int end = kCodes ? K : (K + kStep - 1) / kStep * kStep;
  const int vectors = (end + 7) / 8;

  const u32x4 none = {0u, 0u, 0u, 0u};
  auto load = [&](const uint8_t* p, int k) __attribute__((always_inline)) {
    if constexpr (kWhole) return k < K ? load_whole<T>(p, k) : none;
    else return load_near<T>(p, k, K);
  };
  auto settled = [&](u32x4 v, int k) __attribute__((always_inline)) { return kWhole ? v : settle<T>(v, k, K); };
  // (h goes past the cache where the row stays in registers and is not read back)
  auto store = [&](uint8_t* p, int k, u32x4 v) __attribute__((always_inline)) {
    if (kWhole && k < K) store_bytes<2, (NV > 0)>(p + (int64_t)k * 2, 16, v);
    if (!kWhole) store_vector<T, (NV > 0)>(p, k, K, v);
  };
  // (0 * an infinite or NaN factor: the elements behind K stay 0)
  auto cut = [&](u32x4 v, int k) __attribute__((always_inline)) {
    if (kWhole) return k < K ? v : none;
    if (k + 8 > K) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j >= K) v[j / 2] &= j % 2 ? 0x0000FFFFu : 0xFFFF0000u;
    }
    return v;
  };
  auto sum_of = [&](u32x4 xv, u32x4 rv) __attribute__((always_inline)) {
    if (r == nullptr) return xv;
    float f[8], e[8];
    spread<T>(xv, f);
    spread<T>(rv, e);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += e[i];
    return join<T>(f);
  };
  auto squares = [&](u32x4 h) __attribute__((always_inline)) {
    float f[8];
    spread<T>(h, f);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fma((double)f[i], (double)f[i], s);
    return s;
  };
  auto normed = [&](u32x4 h, u32x4 g, float f) __attribute__((always_inline)) {
    float v[8], e[8];
    spread<T>(h, v);
    spread<T>(g, e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] *= f;
      if (a.gain != nullptr) v[i] *= e[i];
    }
    return join<T>(v);
  };
  auto factor = [&](double sum) __attribute__((always_inline)) { return (float)inverse_root(__builtin_fma(sum, a.inv_k, a.eps)); };
  auto store_codes = [&](int k, u32x4 y, const CodeScale& cs) __attribute__((always_inline)) {
    float f[8];
    spread<T>(y, f);
    const u32x2 c = cs.codes(f, a.q);
    if (k < K) {
      uint8_t* const dst = reinterpret_cast<uint8_t*>(a.codes) + row * K + k;
      store_bytes<1>(dst, kWhole ? 8 : min(K - k, 8), u32x4{c[0], c[1], 0u, 0u});
    }
  };
  // (the four lanes of a block are neighbours, active together)
  auto store_mx4 = [&](int k, u32x4 y) __attribute__((always_inline)) {
    uint32_t m = fold_magnitude<T>(0u, y);
    m = widest<T>(m);
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));
    const uint32_t byte = scale_byte<T>(m);
    const uint32_t c = byte == 255u ? 0u : codes_of<T>(&y, scale_of(byte));
    const int64_t unit = row / kGroup * a.mx.steps + k / kStep;
    const int s = (int)(row % kGroup), b = k % kStep / kBlock;
    *reinterpret_cast<uint32_t*>(a.mx.codes + (unit * 8 + b) * 256 + s * 16 + k % kBlock / 2) = c;
    if (k % kBlock == 0) a.mx.scales[unit * kScaleBytes + b % 2 * 64 + s * 4 + b / 2] = (uint8_t)byte;
  };

  if constexpr (NV > 0) {
    u32x4 v[NV], g[NV];
    {
      u32x4 rv[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = (i * threads + tid) * 8;
        v[i] = load(x, k);
        rv[i] = r != nullptr ? load(r, k) : none;
        g[i] = a.gain != nullptr ? load(a.gain, k) : none;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = (i * threads + tid) * 8;
        v[i] = sum_of(settled(v[i], k), settled(rv[i], k));
        g[i] = settled(g[i], k);
      }
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = (i * threads + tid) * 8;
      if (hrow != nullptr) store(hrow, k, v[i]);
      sum += squares(v[i]);
    }
    const float f = factor(row_sum(sum));
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = (i * threads + tid) * 8;
      v[i] = cut(normed(v[i], g[i], f), k);
      if (yrow != nullptr) store(yrow, k, v[i]);
      if (kCodes) m = fold_magnitude<T>(m, v[i]);
      else if (k < end) store_mx4(k, v[i]);
    }
    if constexpr (kCodes) {
      CodeScale cs;
      cs.set<T>(row_max(widest<T>(m)), a.q);
#pragma unroll
      for (int i = 0; i < NV; ++i) store_codes((i * threads + tid) * 8, v[i], cs);
      if (tid == 0) a.scale[row] = (uint16_t)cs.bits;
    }
  } else {
    auto load_h = [&](int k) __attribute__((always_inline)) {
      const u32x4 xv = load(x, k), rv = r != nullptr ? load(r, k) : none;
      return sum_of(settled(xv, k), settled(rv, k));
    };
    double sum = 0.0;
    for (int i = tid; i < vectors; i += threads) {
      const u32x4 h = load_h(i * 8);
      if (hrow != nullptr) store(hrow, i * 8, h);
      sum += squares(h);
    }
    const float f = factor(row_sum(sum));
    // (h may have replaced x or the residual: it is read back, by the thread that wrote it)
    auto load_y = [&](int k) __attribute__((always_inline)) {
      const u32x4 g = a.gain != nullptr ? load(a.gain, k) : none;
      const u32x4 h = hrow != nullptr ? settled(load(hrow, k), k) : load_h(k);
      return cut(normed(h, settled(g, k), f), k);
    };
    uint32_t m = 0u;
    for (int i = tid; i < vectors; i += threads) {
      const u32x4 y = load_y(i * 8);
      if (yrow != nullptr) store(yrow, i * 8, y);
      if (kCodes) m = fold_magnitude<T>(m, y);
      else store_mx4(i * 8, y);
    }
    if constexpr (kCodes) {
      CodeScale cs;
      cs.set<T>(row_max(widest<T>(m)), a.q);
      for (int i = tid; i < vectors; i += threads) store_codes(i * 8, load_y(i * 8), cs);
      if (tid == 0) a.scale[row] = (uint16_t)cs.bits;
    }
  }
}

// (2 code + 1) scale, eight elements of a row per thread: bound by memory, 1
// byte in and 2 or 4 out per element.  A workgroup takes 2^shift threads' worth of
// 256 >> shift rows: one of `parts` parts of a long row, or several short rows.
struct CodesArgs {
  const int8_t* codes;
  const uint16_t* scale;
  int64_t rows;
  int K, parts, shift;
  uint8_t* out;
};
template <class T, bool kStream>
__global__ __launch_bounds__(256) void dequantize_codes_kernel(CodesArgs a) {
  const int8_t* const codes = a.codes;
  const uint16_t* const scale = a.scale;
  const int K = a.K, parts = a.parts;
  uint8_t* const out = a.out;
  const int64_t row = ((int64_t)(blockIdx.x / (unsigned)parts) << (8 - a.shift)) + (threadIdx.x >> a.shift);
  const int k = ((int)(blockIdx.x % (unsigned)parts << a.shift) + (int)(threadIdx.x & ((1u << a.shift) - 1u))) * 8;
  if (row >= a.rows || k >= K) return;
  const float s = Half::to_float(scale[row]);
  const int8_t* const src = codes + row * K + k;
  typedef uint32_t any_u32x2 __attribute__((ext_vector_type(2), aligned(1)));
  u32x2 c = {0u, 0u};
  if (k + 8 <= K) {
    c = *reinterpret_cast<const any_u32x2*>(src);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < K) c[i / 4] |= (uint32_t)(uint8_t)src[i] << (8 * (i % 4));
  }
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)(2 * (int)(int8_t)(c[i / 4] >> (8 * (i % 4))) + 1) * s;
  uint8_t* const dst = out + row * K * T::kBytes;
  if constexpr (T::kBytes == 4) {
    // (halves of 32 bytes a lane fill their lines in the cache)
    u32x4 lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __builtin_bit_cast(uint32_t, f[i]);
      hi[i] = __builtin_bit_cast(uint32_t, f[4 + i]);
    }
    store_vector<T>(dst, k, K, lo);
    store_vector<T>(dst, k + 4, K, hi);
  } else {
    store_vector<T, kStream>(dst, k, K, join<T>(f));
  }
}

template <class T, bool kCodes, bool kWhole>
hipError_t launch_norm_as(const NormArgs& a, int64_t rows, hipStream_t s) {
  // rows of the launch, by whole groups of 128 for the MX4 mapping
  const unsigned grid = (unsigned)(kCodes ? rows : (rows + 127) / 128 * 128);
  const int vectors = (kCodes ? a.K + 7 : (a.K + kStep - 1) / kStep * kStep) / 8;
  // Many rows of up to 64 vectors: several to a workgroup, with MX4 a group's 16
  // (16384 x 128 into codes 12.0 us with a workgroup each, 5.0 so, 2048 x 300 5.7 and
  // 4.2, 256 x 512 3.0 and 3.3; into MX4 2048 x 300 4.9 and 4.7, 1024 x 512 3.2 and 3.9).
  if (vectors <= 64 && rows >= (kCodes ? 1024 : 2048)) {
    const int lanes = kCodes && vectors <= 16 ? 16 : vectors <= 32 ? 32 : 64;
    const int together = kCodes ? 256 / lanes : kGroup;
    const dim3 blocks((unsigned)((rows + together - 1) / together)), wide((unsigned)(together * lanes));
    if (lanes == 64) return launch_kernel(rmsnorm_kernel<T, 1, 64, kCodes, kWhole>, blocks, wide, 0, s, a);
    if (lanes == 32) return launch_kernel(rmsnorm_kernel<T, 1, 32, kCodes, kWhole>, blocks, wide, 0, s, a);
    if constexpr (kCodes) return launch_kernel(rmsnorm_kernel<T, 1, 16, kCodes, kWhole>, blocks, wide, 0, s, a);
  }
  auto threads = [&](int per) { return dim3((unsigned)((vectors + per * kWave - 1) / (per * kWave) * kWave)); };
  // One vector per thread for few rows (a row alone, 1 x 4096: 3.3 us in a graph
  // against 3.6 with two), two where rows queue and a wave's fixed share of the
  // work counts (2048 x 4096 into codes: 14.1 against 14.6), or are long.
  if (vectors <= 512 && rows < 1024) return launch_kernel(rmsnorm_kernel<T, 1, 0, kCodes, kWhole>, dim3(grid), threads(1), 0, s, a);
  if (vectors <= 2048) return launch_kernel(rmsnorm_kernel<T, 2, 0, kCodes, kWhole>, dim3(grid), threads(2), 0, s, a);
  if (vectors <= 4096) return launch_kernel(rmsnorm_kernel<T, 4, 0, kCodes, kWhole>, dim3(grid), threads(4), 0, s, a);
  return launch_kernel(rmsnorm_kernel<T, 0, 0, kCodes, kWhole>, dim3(grid), dim3(kWave * kMaxWaves), 0, s, a);
}

template <class T, bool kCodes>
hipError_t launch_norm_of(const NormArgs& a, int64_t rows, hipStream_t s) {
  return streams(a.h, a.K, 2) && streams(a.y, a.K, 2) ? launch_norm_as<T, kCodes, true>(a, rows, s)
                                                      : launch_norm_as<T, kCodes, false>(a, rows, s);
}

// A launch holds fewer than 2^32 threads: at 1024 a row, this many rows (whole
// groups of 128).
constexpr int64_t kLaunchRows = (int64_t)1 << 21;

}  // namespace

namespace mx4 {

hipError_t launch_rmsnorm(int M, int K, int type, const void* x, int64_t x_stride, const void* residual, int64_t r_stride,
                          const void* gain, double eps, void* h, void* y, int q, int8_t* codes, uint16_t* scale,
                          const Operand* mx, hipStream_t s) {
  for (int64_t r0 = 0; r0 < M; r0 += kLaunchRows) {
    const int64_t rows = M - r0 < kLaunchRows ? M - r0 : kLaunchRows;
    NormArgs a{};
    a.M = (int)rows;
    a.K = K;
    a.x = static_cast<const uint8_t*>(x) + r0 * x_stride * 2;
    a.x_stride = x_stride;
    if (residual != nullptr) a.residual = static_cast<const uint8_t*>(residual) + r0 * r_stride * 2;
    a.r_stride = r_stride;
    a.gain = static_cast<const uint8_t*>(gain);
    a.inv_k = 1.0 / K;
    a.eps = eps;
    if (h != nullptr) a.h = static_cast<uint8_t*>(h) + r0 * K * 2;
    if (y != nullptr) a.y = static_cast<uint8_t*>(y) + r0 * K * 2;
    a.q = mx == nullptr ? q : 1;
    hipError_t e;
    if (mx == nullptr) {
      a.codes = codes + r0 * K;
      a.scale = scale + r0;
      e = type == APT_TYPE_FP16 ? launch_norm_of<Half, true>(a, rows, s) : launch_norm_of<Bf16, true>(a, rows, s);
    } else {
      a.mx = *mx;
      a.mx.codes += r0 / kGroup * mx->steps * kCodeBytes;
      a.mx.scales += r0 / kGroup * mx->steps * kScaleBytes;
      e = type == APT_TYPE_FP16 ? launch_norm_of<Half, false>(a, rows, s) : launch_norm_of<Bf16, false>(a, rows, s);
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_dequantize_codes(const int8_t* codes, const uint16_t* scale, int M, int K, int type, void* out,
                                   hipStream_t s) {
  const int parts = (K + 2047) / 2048;
  int shift = 0;
  while (shift < 8 && (8 << shift) < K) ++shift;
  const int64_t most = ((int64_t)1 << 23) / parts > 0 ? ((int64_t)1 << 23) / parts : 1;  // rows of a launch
  const int size = type == APT_TYPE_FP32 ? 4 : 2;
  for (int64_t r0 = 0; r0 < M; r0 += most) {
    const int64_t rows = M - r0 < most ? M - r0 : most;
    const dim3 grid((unsigned)((((rows - 1) >> (8 - shift)) + 1) * parts)), block(256);
    const CodesArgs a{codes + r0 * K, scale + r0, rows, K, parts, shift, static_cast<uint8_t*>(out) + r0 * K * size};
    const bool stream = streams_values(a.out, rows, K, size);
    hipError_t e;
    switch (type) {
      case APT_TYPE_FP16:
        e = launch_kernel(stream ? dequantize_codes_kernel<Half, true> : dequantize_codes_kernel<Half, false>, grid, block,
                          0, s, a);
        break;
      case APT_TYPE_BF16:
        e = launch_kernel(stream ? dequantize_codes_kernel<Bf16, true> : dequantize_codes_kernel<Bf16, false>, grid, block,
                          0, s, a);
        break;
      default: e = launch_kernel(dequantize_codes_kernel<Float, false>, grid, block, 0, s, a); break;
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mx4
}  // namespace apt
