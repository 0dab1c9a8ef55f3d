// mx4_gemm.hip - C = A * W^T of two MX4 operands on the block-scaled MFMA, for
// gfx950: the choice among the kernels of mx4_thin.h and mx4_tile.h, and their
// launches.
#include <algorithm>
#include <cmath>

#include "mx4_thin.h"

namespace apt {
namespace {

using namespace mx4;

// A tile shape and what a step of 256 elements of K costs a workgroup of it, in
// us: with few compute units busy, with each running one (in between in
// proportion: what they share, clock, caches and memory, counts long before the
// chip is full), and its share where each runs several.  `fixed`: what it needs
// besides more than the others.  Measured at bf16 output on 64 to 2048 rows by
// 4096 and 11008 columns, K = 4096 to 11008.
struct Tile {
  int mb, nb;
  double few, one, share, fixed;
};
constexpr Tile kTiles[] = {
    {1, 1, 0.22, 0.25, 0.25, 0.0},  // 32 x 128
    {2, 1, 0.25, 0.34, 0.31, 0.0},  // 64 x 128
    {4, 1, 0.36, 0.50, 0.55, 0.0},  // 128 x 128
    {4, 2, 0.32, 1.00, 0.84, 0.0},  // 128 x 256
    {8, 2, 0.85, 1.60, 1.60, 4.0},  // 256 x 256, one workgroup per compute unit: its epilogue stands alone
};
constexpr int kNumTiles = sizeof(kTiles) / sizeof(kTiles[0]);
constexpr double kUnits = 256.0;  // compute units

// Activations given as rows are quantized by the few-row kernel's workgroups
// themselves, each on its own, up to this many elements (rows padded to steps).
// The conversion takes 0.8 us per 4096 elements and saves a launch, which is 1.5 us
// of a graph and 4 us of a call's time on the host.  Fused and not, in a graph: 1 x
// 11008 x 4096 6.1 and 8.4 us, 2 x 11008 x 4096 6.9 and 8.5, 3 x 11008 x 4096 8.1 and 8.4,
// 4 x 11008 x 4096 9.2 and 8.5 (called by itself 8.7 and 11.0), 4 x 4096 x 4096 5.4 and 5.2
// (7.0 and 10.9), 6 x 4096 x 4096 7.2 and 5.4, 16 x 4096 x 1024 5.5 and 5.2 (7.1 and 11.1).
constexpr int64_t kFusedElements = 16384;

int64_t tiles_of(int M, int N, const Tile& t) {
  return ((int64_t)M + t.mb * 32 - 1) / (t.mb * 32) * (((int64_t)N + t.nb * 128 - 1) / (t.nb * 128));
}

double per_step(double tiles, const Tile& t) {
  const double load = tiles / kUnits;
  return load <= 1.0 ? t.few + (t.one - t.few) * load : t.share * std::ceil(load);
}

// Workgroups of the few-row kernel at mt groups of 16 activation rows each.
int64_t thin_blocks(int M, int N, int mt) { return ((int64_t)M + 16 * mt - 1) / (16 * mt) * groups(N); }

// Its time in us.  A compute unit takes in about 105 bytes a ns, and a workgroup
// reads 16 weight rows and 16 mt activation rows of 136 bytes a step; one alone is
// bound by the loads' latency.  Weights from memory count by a third: the rest
// hides.  Measured on 16 to 512 rows by 128 to 11008 columns, K = 1024 to 11008.
double thin_time(int M, int N, int K, int mt) {
  const double S = steps(K), load = (double)thin_blocks(M, N, mt) / kUnits;
  const double few = 0.011 + 0.0175 * mt, one = 0.0207 * (mt + 1);
  const double per = load <= 1.0 ? few + (one - few) * load : one * std::ceil(load);
  return 2.4 + 0.05 * mt * std::ceil(load) + S * per + 0.3 * N * (double)K * 17 / 32 / 5.2e6;
}

// The kernel of a problem: -mt for the few-row kernel, else an index into kTiles.
// Up to 32 rows the few-row kernel is the faster everywhere (32 x 11008 x 4096
// 6.8 us against 7.7, 32 x 4096 x 11008 6.6 against 14.7); beyond, the modelled times
// decide.  It wins where its 16 columns a workgroup fill the chip and the tiles' 128 do
// not (64 x 512 x 11008 3.7 us at mt = 1, 4.6 and 6.5 at 2 and 4, tiles 9; 256 x 512 x
// 11008 5.9 at mt = 2, tiles 11.9; 128 x 2048 x 11008 8.1 at mt = 4, tiles 12.3; 128 x 4096
// x 11008 13.4 at mt = 4, tiles 12.6; 64 x 11008 x 4096 9.3 at mt = 4, tiles 7.2).  Among
// the tiles a large one costs fewer loads per MFMA and a small one fills the chip:
// 2048 x 11008 x 4096 takes 46 us at 128 x 256 and 59, 56, 64, 90 at 256 x 256,
// 128, 64 and 32 x 128; 333 x 5003 x 2999 7.3 us at 64 x 128, 9.1 and 11.9 at 128 x
// 128 and 128 x 256; 1024 x 4096 x 11008 25 at 128 x 128 and 31 at 128 x 256.
int kernel_of(int M, int N, int K) {
  int best = -1;
  double least = thin_time(M, N, K, 1);
  auto consider = [&](int kernel, double us) {
    if (us < least) {
      least = us;
      best = kernel;
    }
  };
  if (M > 16) consider(-2, thin_time(M, N, K, 2));
  if (M <= 32) return best;
  consider(-4, thin_time(M, N, K, 4));
  for (int i = 0; i < kNumTiles; ++i) {
    const Tile& t = kTiles[i];
    consider(i, 1.9 + steps(K) * per_step((double)tiles_of(M, N, t), t) + t.fixed);
  }
  return best;
}

template <class T, int I>
hipError_t launch_tile(GemmParams p, hipStream_t s) {
  constexpr int MB = kTiles[I].mb, NB = kTiles[I].nb;
  // (registers: four steps of weights where the accumulators leave room)
  constexpr int WD = NB == 1 ? 4 : 2;
  p.tiles_m = (int)(((int64_t)p.M + MB * 32 - 1) / (MB * 32));
  p.tiles_n = (int)(((int64_t)p.N + NB * 128 - 1) / (NB * 128));
  const dim3 grid((unsigned)(p.tiles_m * p.tiles_n)), block(kWave * kTileWaves);
  return launch_kernel(tile_kernel<T, MB, NB, WD>, grid, block, 0, s, p);
}

template <class T>
hipError_t launch_tile_of(const GemmParams& p, int kernel, hipStream_t s) {
  switch (kernel) {
    case 0: return launch_tile<T, 0>(p, s);
    case 1: return launch_tile<T, 1>(p, s);
    case 2: return launch_tile<T, 2>(p, s);
    case 3: return launch_tile<T, 3>(p, s);
    default: return launch_tile<T, 4>(p, s);
  }
}

hipError_t launch_thin(const ThinParams& p, int mt, hipStream_t s) {
  const dim3 grid((unsigned)thin_blocks(p.M, p.N, mt)), block(kWave * kThinWaves);
  switch (mt) {
    case 1: return launch_kernel(thin_kernel<1, void>, grid, block, 0, s, p);
    case 2: return launch_kernel(thin_kernel<2, void>, grid, block, 0, s, p);
    default: return launch_kernel(thin_kernel<4, void>, grid, block, 0, s, p);
  }
}

}  // namespace

namespace mx4 {

int64_t gemm_tiles(int M, int N, int K) {
  const int k = kernel_of(M, N, K);
  return k < 0 ? thin_blocks(M, N, -k) : tiles_of(M, N, kTiles[k]);
}

hipError_t launch_gemm(int M, int N, int K, const Operand& a, const Operand& w, int type, void* c, hipStream_t s) {
  const int k = kernel_of(M, N, K);
  if (k < 0) return launch_thin(ThinParams{M, N, type, w.steps, a, w, static_cast<uint8_t*>(c), nullptr, 0, K}, -k, s);
  const GemmParams p{M, N, a, w, static_cast<uint8_t*>(c), 0, 0};
  switch (type) {
    case APT_TYPE_FP16: return launch_tile_of<Half>(p, k, s);
    case APT_TYPE_BF16: return launch_tile_of<Bf16>(p, k, s);
    default: return launch_tile_of<Float>(p, k, s);
  }
}

bool gemm_takes_rows(int M, int K) { return M <= 16 && (int64_t)M * steps(K) * kStep <= kFusedElements; }

hipError_t launch_gemm_rows(int M, int N, int K, const void* x, int x_type, int64_t x_stride, const Operand& w, int type,
                            void* c, hipStream_t s) {
  const ThinParams p{M, N, type, w.steps, Operand{}, w, static_cast<uint8_t*>(c), static_cast<const uint8_t*>(x), x_stride, K};
  const dim3 grid((unsigned)w.groups), block(kWave * kThinWaves);
  const size_t lds = thin_lds_bytes(M, K);
  switch (x_type) {
    case APT_TYPE_FP16: return launch_kernel(thin_kernel<1, Half>, grid, block, lds, s, p);
    case APT_TYPE_BF16: return launch_kernel(thin_kernel<1, Bf16>, grid, block, lds, s, p);
    default: return launch_kernel(thin_kernel<1, Float>, grid, block, lds, s, p);
  }
}

}  // namespace mx4
}  // namespace apt
