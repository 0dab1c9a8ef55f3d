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
// chip is full), and its share where each runs several.  A launch with its first
// loads and its outputs takes kTileEnds besides, and `fixed` more.  Measured at
// bf16 output on 64 to 2048 rows by 4096 to 28672 columns, K = 4096 to 11008.
struct Tile {
  int mb, nb;
  double few, one, share, fixed;
};
constexpr Tile kTiles[] = {
    {1, 1, 0.22, 0.25, 0.25, 0.0},  // 32 x 128
    {2, 1, 0.25, 0.34, 0.331, 0.0},  // 64 x 128
    {4, 1, 0.36, 0.50, 0.55, 0.0},  // 128 x 128
    {4, 2, 0.32, 1.00, 0.84, 0.0},  // 128 x 256
    {8, 2, 0.85, 1.60, 1.60, 4.0},  // 256 x 256, one workgroup per compute unit: its epilogue stands alone
};
constexpr int kNumTiles = sizeof(kTiles) / sizeof(kTiles[0]);
constexpr double kTileEnds = 1.9;
constexpr double kUnits = 256.0;  // compute units

// Activations given as rows are quantized by the few-row kernel's workgroups
// themselves, each on its own, up to kFusedElements elements (rows padded to steps)
// where that is the faster way.
// The conversion takes 0.8 us per 4096 elements and saves a launch, which is 1.5 us
// of a graph and 4 to 5 us of a call's time on the host.  Fused and not, in a graph
// and by itself: 1 x 11008 x 4096 6.2 and 8.5, 7.3 and 12.5 us; 3 x 11008 x 4096 7.9 and 8.5, 7.6
// and 12.5; 4 x 11008 x 4096 8.8 and 8.4, 8.5 and 12.4; 4 x 4096 x 4096 5.4 and 5.2, 7.2 and
// 12.2; 16 x 4096 x 1024 5.4 and 5.1, 7.2 and 12.4; 6 x 4096 x 4096 7.2 and 5.4 in a graph.
// Every 16 weight rows repeat it, so with many of them it costs more than a launch
// either way: from kFusedRows on, it ends at kFusedWork elements times groups (4 x
// 16384 x 4096 10.7 and 10.0, 10.4 and 12.4; 4 x 24576 x 4096 14.2 and 12.3, 13.9 and 12.6;
// 4 x 32000 x 4096 17.0 and 14.4, 16.7 and 13.9; 16 x 32000 x 1024 12.9 and 9.4, 12.3 and
// 12.3).  One or two rows' conversion hides behind the weights at any N (2 x 64000 x
// 4096 22.8 and 24.8, 22.1 and 23.9; 2 x 64000 x 8192 51.7 and 51.0, 47.5 and 48.2).
constexpr int64_t kFusedElements = 16384;
constexpr int kFusedRows = 3;
constexpr int64_t kFusedWork = (int64_t)1 << 24;

int64_t tiles_of(int M, int N, const Tile& t) {
  return ((int64_t)M + t.mb * 32 - 1) / (t.mb * 32) * (((int64_t)N + t.nb * 128 - 1) / (t.nb * 128));
}

double per_step(double tiles, const Tile& t) {
  const double load = tiles / kUnits;
  return load <= 1.0 ? t.few + (t.one - t.few) * load : t.share * std::ceil(load);
}

// A workgroup of the few-row kernel: 16 mt activation rows by 16 nt weight rows, the
// steps it holds of each, and its time in us: `fixed` and `turn` for its start and
// end, alone and for each that a compute unit runs in turn; a step of 256 elements
// costs `few` with few units busy (loads' latency), `one` with each running one,
// and `share` with several (a unit takes in about 105 bytes a ns, and a step is
// 2176 (mt + nt)).  Measured on 16 to 768 rows by 128 to 11008 columns, K = 1024 to
// 11008.  (64 x 16 rows come behind 32 x 32 everywhere, 64 x 64 behind one of these
// or a tile.)
struct Thin {
  int mt, nt, ka, da;
  double fixed, turn, few, one, share;
};
constexpr Thin kThins[] = {
    {1, 1, 4, 4, 2.4, 0.05, 0.028, 0.041, 0.041},
    {2, 1, 4, 4, 2.4, 0.10, 0.046, 0.062, 0.062},
    {2, 2, 4, 4, 2.7, 0.25, 0.067, 0.088, 0.083},
    {4, 2, 2, 2, 3.6, 0.40, 0.100, 0.125, 0.115},
};
constexpr int kNumThins = sizeof(kThins) / sizeof(kThins[0]);

int64_t blocks_of(int M, int N, const Thin& t) {
  return ((int64_t)M + 16 * t.mt - 1) / (16 * t.mt) * ((groups(N) + t.nt - 1) / t.nt);
}

double thin_time(int M, int N, int K, const Thin& t) {
  const double load = (double)blocks_of(M, N, t) / kUnits, turns = std::ceil(load);
  return t.fixed + t.turn * turns + steps(K) * (load <= 1.0 ? t.few + (t.one - t.few) * load : t.share * turns);
}

// The kernel of a problem: an index into kThins, or kNumThins and more for kTiles.
// Up to 32 rows the few-row kernel is the faster everywhere (32 x 11008 x 4096
// 6.8 us against 7.7, 32 x 4096 x 11008 6.6 against 14.7); beyond, the modelled times
// decide.  It wins where tiles of 128 columns leave much of the chip idle (in us, the
// four workgroups of kThins and the best tile: 64 x 512 x 11008 3.7, 4.6, 5.9, 8.3, 9;
// 64 x 4096 x 11008 11.6, 9.3, 7.7, 10.1, 12.5; 256 x 1024 x 11008 10.0, 8.5, 7.4, 9.7, 12.3; 128 x
// 4096 x 11008 19.1, 15.1, 11.4, 10.3, 12.5; 256 x 4096 x 11008 34, 26, 18.8, 15.8, 13.3).  Among
// the tiles a large one costs fewer loads per MFMA and a small one fills the chip:
// 2048 x 11008 x 4096 takes 46 us at 128 x 256 and 58, 56, 64, 90 at 256 x 256,
// 128, 64 and 32 x 128; 333 x 5003 x 2999 7.3 us at 64 x 128, 9.1 and 11.9 at 128 x
// 128 and 128 x 256; 1024 x 4096 x 11008 25 at 128 x 128 and 31 at 128 x 256.
int kernel_of(int M, int N, int K) {
  int best = 0;
  double least = thin_time(M, N, K, kThins[0]);
  auto consider = [&](int kernel, double us) {
    if (us < least) {
      least = us;
      best = kernel;
    }
  };
  for (int i = 1; i < kNumThins; ++i)
    if (M > 8 * kThins[i].mt) consider(i, thin_time(M, N, K, kThins[i]));
  if (M <= 32) return best;
  for (int i = 0; i < kNumTiles; ++i) {
    const Tile& t = kTiles[i];
    consider(kNumThins + i, kTileEnds + steps(K) * per_step((double)tiles_of(M, N, t), t) + t.fixed);
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

template <int I>
hipError_t launch_thin(const ThinParams& p, hipStream_t s) {
  constexpr Thin t = kThins[I];
  const dim3 grid((unsigned)blocks_of(p.M, p.N, t)), block(kWave * kThinWaves);
  return launch_kernel(thin_kernel<t.mt, t.nt, t.ka, t.da, void>, grid, block, 0, s, p);
}

hipError_t launch_thin_of(const ThinParams& p, int kernel, hipStream_t s) {
  switch (kernel) {
    case 0: return launch_thin<0>(p, s);
    case 1: return launch_thin<1>(p, s);
    case 2: return launch_thin<2>(p, s);
    default: return launch_thin<3>(p, s);
  }
}

}  // namespace

namespace mx4 {

int64_t gemm_tiles(int M, int N, int K) {
  const int k = kernel_of(M, N, K);
  return k < kNumThins ? blocks_of(M, N, kThins[k]) : tiles_of(M, N, kTiles[k - kNumThins]);
}

void gemm_block(int M, int N, int K, int* rows, int* columns) {
  const int k = kernel_of(M, N, K);
  *rows = k < kNumThins ? 16 * kThins[k].mt : 32 * kTiles[k - kNumThins].mb;
  *columns = k < kNumThins ? 16 * kThins[k].nt : 128 * kTiles[k - kNumThins].nb;
}

hipError_t launch_gemm(int M, int N, int K, const Operand& a, const Operand& w, int type, void* c, hipStream_t s) {
  const int k = kernel_of(M, N, K);
  if (k < kNumThins)
    return launch_thin_of(ThinParams{M, N, type, w.steps, a, w, static_cast<uint8_t*>(c), nullptr, 0, K}, k, s);
  const GemmParams p{M, N, a, w, static_cast<uint8_t*>(c), 0, 0};
  switch (type) {
    case APT_TYPE_FP16: return launch_tile_of<Half>(p, k - kNumThins, s);
    case APT_TYPE_BF16: return launch_tile_of<Bf16>(p, k - kNumThins, s);
    default: return launch_tile_of<Float>(p, k - kNumThins, s);
  }
}

bool gemm_takes_rows(int M, int K) { return M <= 16 && (int64_t)M * steps(K) * kStep <= kFusedElements; }
bool gemm_prefers_rows(int M, int N, int K) {
  return gemm_takes_rows(M, K) && (M < kFusedRows || (int64_t)M * steps(K) * kStep * groups(N) <= kFusedWork);
}

hipError_t launch_gemm_rows(int M, int N, int K, const void* x, int x_type, int64_t x_stride, const Operand& w, int type,
                            void* c, hipStream_t s) {
  const ThinParams p{M, N, type, w.steps, Operand{}, w, static_cast<uint8_t*>(c), static_cast<const uint8_t*>(x), x_stride, K};
  const dim3 grid((unsigned)w.groups), block(kWave * kThinWaves);
  const size_t lds = thin_lds_bytes(M, K);
  switch (x_type) {
    case APT_TYPE_FP16: return launch_kernel(thin_kernel<1, 1, 4, 2, Half>, grid, block, lds, s, p);
    case APT_TYPE_BF16: return launch_kernel(thin_kernel<1, 1, 4, 2, Bf16>, grid, block, lds, s, p);
    default: return launch_kernel(thin_kernel<1, 1, 4, 2, Float>, grid, block, lds, s, p);
  }
}

}  // namespace mx4
}  // namespace apt
