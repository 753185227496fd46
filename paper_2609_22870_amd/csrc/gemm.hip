// Scaled FP8 GEMM of the FP8 linear layer on gfx950: the kernels and their
// launches (gemm_tile.h has what a workgroup does).
#include "gemm_tile.h"

namespace fp8q {

namespace gemm_detail {

template <int PAIR, int TI, int TJ, bool QOUT, int FMT>
__global__ __launch_bounds__(kThinWaves * 64) void gemm_thin_kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[ThinLds<TI, TJ>::kBytes];
  int tm, tn;
  tile_coords<TI * 16, TJ * 16>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  thin_tile<PAIR, TI, TJ, QOUT, FMT>(g, lds, tm, tn);
}

template <int PAIR, int BM, int BN, int WM, int WN, bool QOUT, int FMT, int KS = 1, int SUMS = 1>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64 * KS) void gemm_kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<PAIR, BM, BN, WM, WN, KS>::kBytes];
  int tm, tn;
  tile_coords<BM, BN>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  gemm_tile<PAIR, BM, BN, WM, WN, QOUT, FMT, KS, false, SUMS>(g, lds, tm, tn);
}

// Large problems: 256 x 256 tiles, one per CU at a time, so the launch runs
// in rounds of kCUs tiles and a last round with few tiles leaves most of the
// chip idle for a whole tile's time.  The workgroups past `full` (a multiple
// of kCUs, or every tile) therefore take a part of a tile each: the tiles at
// raster positions full, full + 1, ... are cut into `parts` = 4 of 128 x 128
// (eight waves of 32 x 64) or 2 of 128 x 256 (eight waves of 64 x 64), which
// run on 4 or 2 times as many CUs for 0.34 or 0.59 of a tile's time (one round
// of each at K = 4096: 19, 33 and 56 us; blockwise 3001 x 5120 x 17408, 3.2
// rounds, 268 -> 242 us; power-of-two scales 4096 x 5120 x 17408, 4.25 rounds,
// 321 -> 301 us; 2048 x 4096 x 12288, 1.5 rounds, 105 us on 128 x 128 tiles ->
// 95 us).  Every tile shape sums an output's K blocks in the
// same order, so the cut changes no bit.

template <int PAIR>
struct LargeLds {
  static constexpr int kWhole = TileLds<PAIR, 256, 256, 128, 64>::kBytes, kHalf = TileLds<PAIR, 128, 256, 64, 64>::kBytes,
                       kQuarter = TileLds<PAIR, 128, 128, 32, 64>::kBytes;
  static constexpr int kMost = kWhole > kHalf ? kWhole : kHalf;
  static constexpr int kBytes = kMost > kQuarter ? kMost : kQuarter;
};

// at(position, g, tm, tn): the problem and 256 x 256 tile of a raster position
template <int PAIR, bool QOUT, int FMT, typename At>
__device__ __forceinline__ void large_tiles(uint8_t* lds, int full, int parts, At&& at) {
  const int b = blockIdx.x;
  const GemmArgs* g;
  int tm, tn;
  if (b < full) {
    at(xcd_order(full, b), g, tm, tn);
    gemm_tile<PAIR, 256, 256, 128, 64, QOUT, FMT>(*g, lds, tm, tn);
    return;
  }
  const int t = xcd_order((int)gridDim.x - full, b - full);  // (full % 8 == 0: the XCD is still b % 8)
  const int part = t & (parts - 1);
  at(full + (parts == 4 ? t >> 2 : t >> 1), g, tm, tn);
  tm = 2 * tm + (part & 1);
  if ((int64_t)tm * 128 >= g->M) return;  // (the whole workgroup: a part past the edge of C)
  if (parts == 4) {
    tn = 2 * tn + (part >> 1);
    if ((int64_t)tn * 128 >= g->N) return;
    gemm_tile<PAIR, 128, 128, 32, 64, QOUT, FMT>(*g, lds, tm, tn);
  } else {
    gemm_tile<PAIR, 128, 256, 64, 64, QOUT, FMT>(*g, lds, tm, tn);
  }
}

template <int PAIR, bool QOUT, int FMT>
__global__ __launch_bounds__(512) void gemm_large_kernel(GemmArgs args, int full, int parts) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[LargeLds<PAIR>::kBytes];
  large_tiles<PAIR, QOUT, FMT>(lds, full, parts, [&](int id, const GemmArgs*& g, int& tm, int& tn) {
    g = &args;
    raster<256, 256>(args.M, args.N, args.K, id, tm, tn);
  });
}

// Split-K: g.splits workgroups per 128 x 128 tile.  Positions run split by
// split over the tile raster, so the tiles of one split (which share the A
// rows of its K range) sit on neighbouring XCDs, and the two tile rows of
// a 256-row problem that share B rows on one XCD.
template <int PAIR, int BM, int BN, int WM, int WN, int FMT>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void gemm_splitk_kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<PAIR, BM, BN, WM, WN>::kBytes];
  const int tiles = (int)((g.M + BM - 1) / BM) * (int)((g.N + BN - 1) / BN);
  const int id = xcd_order(tiles * g.splits, blockIdx.x);
  const int split = id / tiles, t = id - split * tiles;
  int tm, tn;
  raster<BM, BN>(g.M, g.N, g.K, t, tm, tn);
  gemm_tile<PAIR, BM, BN, WM, WN, false, FMT, 1, true>(g, lds, tm, tn, split, t);
}

// Grouped GEMM: one launch over several problems that share the pair, the
// formats and K (the fused QKV or gate / up projections: one activation
// operand, several weights and outputs).  The workgroups' XCD-ordered
// positions run over the problems' rasters one after another; the problem
// of a position is found from the prefix sums of the tile counts.
template <int BM, int BN>
__device__ __forceinline__ const GemmArgs* grouped_at(const GemmGroup& gs, int id, int& tm, int& tn) {
  int p = 0;
  for (int i = 1; i < gs.count; ++i) p += id >= gs.tile_start[i] ? 1 : 0;
  raster<BM, BN>(gs.prob[p].M, gs.prob[p].N, gs.prob[p].K, id - gs.tile_start[p], tm, tn);
  return &gs.prob[p];
}

template <int PAIR, int BM, int BN, int WM, int WN, int KS = 1>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64 * KS) void gemm_grouped_kernel(GemmGroup gs) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<PAIR, BM, BN, WM, WN, KS>::kBytes];
  int tm, tn;
  const GemmArgs* g = grouped_at<BM, BN>(gs, xcd_order(gs.tile_start[gs.count], blockIdx.x), tm, tn);
  gemm_tile<PAIR, BM, BN, WM, WN, false, 0, KS>(*g, lds, tm, tn);
}

template <int PAIR, int TI, int TJ>
__global__ __launch_bounds__(kThinWaves * 64) void gemm_grouped_thin_kernel(GemmGroup gs) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[ThinLds<TI, TJ>::kBytes];
  int tm, tn;
  const GemmArgs* g = grouped_at<TI * 16, TJ * 16>(gs, xcd_order(gs.tile_start[gs.count], blockIdx.x), tm, tn);
  thin_tile<PAIR, TI, TJ, false, 0>(*g, lds, tm, tn);
}

// Problems with two K groups and thin ones in one launch (both sum orders are
// their own, so neither can take the other's kernel): the first workgroups
// take 64 x 64 tiles of `grouped`, the rest 64 x 64 thin tiles of `thin`.
template <int PAIR>
__global__ __launch_bounds__(512) void gemm_grouped_mixed_kernel(GemmGroup grouped, GemmGroup thin) {
  constexpr int kGrouped = TileLds<PAIR, 64, 64, 32, 32, 2>::kBytes, kThin = ThinLds<4, 4>::kBytes;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kGrouped > kThin ? kGrouped : kThin];
  const int first = grouped.tile_start[grouped.count], b = blockIdx.x;
  int tm, tn;
  if (b < first) {
    const GemmArgs* g = grouped_at<64, 64>(grouped, xcd_order(first, b), tm, tn);
    gemm_tile<PAIR, 64, 64, 32, 32, false, 0, 2>(*g, lds, tm, tn);
  } else {
    const GemmArgs* g = grouped_at<64, 64>(thin, xcd_order(thin.tile_start[thin.count], b - first), tm, tn);
    thin_tile<PAIR, 4, 4, false, 0>(*g, lds, tm, tn);
  }
}

template <int PAIR>
__global__ __launch_bounds__(512) void gemm_grouped_large_kernel(GemmGroup gs, int full, int parts) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[LargeLds<PAIR>::kBytes];
  large_tiles<PAIR, false, 0>(lds, full, parts, [&](int id, const GemmArgs*& g, int& tm, int& tn) {
    g = grouped_at<256, 256>(gs, id, tm, tn);
  });
}

template <int PAIR, int BM, int BN, int WM, int WN, bool QOUT, int FMT, int KS = 1, int SUMS = 1>
hipError_t launch_tiles(const GemmArgs& g, hipStream_t s) {
  const int64_t tiles = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
  constexpr int threads = (BM / WM) * (BN / WN) * 64 * KS;
  gemm_kernel<PAIR, BM, BN, WM, WN, QOUT, FMT, KS, SUMS><<<dim3((unsigned)tiles), threads, 0, s>>>(g);
  return hipGetLastError();
}

template <int PAIR, bool QOUT, int FMT>
hipError_t launch_large(const GemmArgs& g, hipStream_t s) {
  const int64_t tiles = ((g.M + 255) / 256) * ((g.N + 255) / 256);
  if (tiles <= 0 || tiles > 0x3fffffff) return hipErrorInvalidValue;
  const LargePlan p = large_plan(tiles);
  gemm_large_kernel<PAIR, QOUT, FMT><<<dim3((unsigned)p.grid), 512, 0, s>>>(g, p.full, p.parts);
  return hipGetLastError();
}

// f(TI, TJ) of a thin tile, as integral constants.
template <typename F>
hipError_t with_thin(int config, F&& f) {
  using std::integral_constant;
  switch (config) {
    case kThin16x16: return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    case kThin16x32: return f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    case kThin32x32: return f(integral_constant<int, 2>{}, integral_constant<int, 2>{});
    case kThin32x64: return f(integral_constant<int, 2>{}, integral_constant<int, 4>{});
    case kThin64x64: return f(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    default: return hipErrorInvalidValue;
  }
}

inline GemmSize size_of(const GemmArgs& g) { return GemmSize{g.M, g.N, g.K}; }

template <int PAIR, bool QOUT, int FMT>
hipError_t launch_thin(const GemmArgs& g, hipStream_t s) {
  auto launch = [&](auto ti, auto tj) {
    constexpr int TI = decltype(ti)::value, TJ = decltype(tj)::value;
    const int64_t tiles = ((g.M + TI * 16 - 1) / (TI * 16)) * ((g.N + TJ * 16 - 1) / (TJ * 16));
    if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
    gemm_thin_kernel<PAIR, TI, TJ, QOUT, FMT><<<dim3((unsigned)tiles), kThinWaves * 64, 0, s>>>(g);
    return hipGetLastError();
  };
  if constexpr (QOUT) {
    return launch(std::integral_constant<int, 2>{}, std::integral_constant<int, 8>{});
  } else {
    const GemmSize size = size_of(g);
    double ns;
    return with_thin(thin_config(&size, 1, ns), launch);
  }
}

template <int PAIR, bool QOUT, int FMT>
hipError_t launch_pair(const GemmArgs& g, hipStream_t s) {
  switch (QOUT ? gemm_quantized_route(size_of(g)) : gemm_route(PAIR, size_of(g))) {
    case kLargeTiles: return launch_large<PAIR, QOUT, FMT>(g, s);
    case kMidTiles: return launch_tiles<PAIR, 128, 128, 64, 64, QOUT, FMT>(g, s);
    case kEightWaves: return launch_tiles<PAIR, 128, 128, 32, 64, QOUT, FMT>(g, s);
    case kThinTiles: return launch_thin<PAIR, QOUT, FMT>(g, s);
    case kTwoKGroups:
      if constexpr (QOUT)
        return launch_tiles<PAIR, 128, 128, 32, 64, QOUT, FMT, 1, 2>(g, s);
      else
        return launch_tiles<PAIR, 64, 64, 32, 32, QOUT, FMT, 2>(g, s);
    case kSmallTiles:
      if constexpr (!QOUT) return launch_tiles<PAIR, 64, 64, 32, 32, QOUT, FMT>(g, s);
      break;
    default: break;
  }
  return hipErrorInvalidValue;
}

// The kernels address operands with 32-bit offsets: split the problem into
// sub-GEMMs whose A and B row ranges each span less than 4 GiB.
template <int PAIR, bool QOUT, int FMT>
hipError_t launch_split(const GemmArgs& g, hipStream_t s) {
  // 32-bit offsets: each sub-problem's A rows, B rows and C rows span
  // < 2 GiB, and row / column indices stay below 2^31 / 4
  const int64_t lim = (int64_t)1 << 31;
  int64_t mstep = g.M, nstep = g.N;
  if (g.M * g.lda >= lim) mstep = ((lim - 1) / g.lda) / 256 * 256;
  // (quantized output is cut where fp8q_gemm with contiguous C, ldc = N, is:
  // the last cut's kernel, and so its K sums, are then the plain call's)
  const int64_t c_row_bytes = QOUT && g.ldq > 2 * g.ldc ? g.ldq : 2 * g.ldc;
  if (g.M * c_row_bytes >= lim) {
    const int64_t cstep = ((lim - 1) / c_row_bytes) / 256 * 256;
    if (cstep < mstep) mstep = cstep;
  }
  // column steps in whole 2048-column pairs of bands, so that a
  // sub-problem's tiles take the K direction of their global columns
  // (odd 1024-column bands walk K backwards)
  if (g.N * g.ldb >= lim) {
    const int64_t q = (lim - 1) / g.ldb;
    nstep = q >= 2048 ? q / 2048 * 2048 : q / 256 * 256;
  }
  if (mstep > ((int64_t)1 << 28)) mstep = (int64_t)1 << 28;
  if (nstep > ((int64_t)1 << 28)) nstep = (int64_t)1 << 28;
  if (mstep <= 0 || nstep <= 0) return hipErrorInvalidValue;
  for (int64_t m = 0; m < g.M; m += mstep) {
    for (int64_t n = 0; n < g.N; n += nstep) {
      GemmArgs sub = g;
      sub.M = (g.M - m) < mstep ? (g.M - m) : mstep;
      sub.N = (g.N - n) < nstep ? (g.N - n) : nstep;
      sub.A = g.A + m * g.lda;
      sub.B = g.B + n * g.ldb;
      if (QOUT) {
        sub.Cq = g.Cq + m * g.ldq + n;
        sub.Cs = g.Cs + (n / 128) * g.cs_ld + m;  // n is a multiple of 256
      } else {
        sub.C = g.C + m * g.ldc + n;
      }
      // scale arrays keep the full problem's layout (strides sa_ld, sb_ld);
      // re-base them at the sub-problem's first row / column
      int64_t da = 0, db = 0;
      if (PAIR != kPairTensor) da = m;
      if (PAIR == kPairRow || PAIR == kPairBlockK) db = n;
      if (PAIR == kPairBlock || PAIR == kPairBlockE8) db = (n / 128) * (g.K / 128);
      sub.sA = g.sA + da;
      sub.sB = g.sB + db;
      sub.sa_count = g.sa_count - da;
      sub.sb_count = g.sb_count - db;
      hipError_t e = launch_pair<PAIR, QOUT, FMT>(sub, s);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

// Explicit instantiations: the host pass otherwise emits launch stubs only
// for the first instantiated pair.
#define FP8Q_GEMM_KERNEL(PAIR, BM, BN, WM, WN) \
  template __global__ void gemm_kernel<PAIR, BM, BN, WM, WN, false, 0>(GemmArgs);
// the backward pairs with E5M2 operands (formats 1, 2, 3)
#define FP8Q_GEMM_KERNEL_FMT(PAIR, BM, BN, WM, WN)                               \
  template __global__ void gemm_kernel<PAIR, BM, BN, WM, WN, false, 1>(GemmArgs); \
  template __global__ void gemm_kernel<PAIR, BM, BN, WM, WN, false, 2>(GemmArgs); \
  template __global__ void gemm_kernel<PAIR, BM, BN, WM, WN, false, 3>(GemmArgs);
FP8Q_GEMM_KERNEL(kPairTensor, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL(kPairRow, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL(kPairBlock, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL(kPairBlockK, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL(kPairTensor, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL(kPairRow, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL(kPairBlock, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL(kPairBlockK, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL(kPairBlockE8, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL(kPairTensor, 64, 64, 32, 32)
FP8Q_GEMM_KERNEL(kPairRow, 64, 64, 32, 32)
FP8Q_GEMM_KERNEL(kPairBlock, 64, 64, 32, 32)
FP8Q_GEMM_KERNEL(kPairBlockK, 64, 64, 32, 32)
FP8Q_GEMM_KERNEL(kPairBlockE8, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL(kPairBlockE8, 64, 64, 32, 32)
FP8Q_GEMM_KERNEL_FMT(kPairBlock, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL_FMT(kPairBlock, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL_FMT(kPairBlockK, 128, 128, 32, 64)
FP8Q_GEMM_KERNEL_FMT(kPairBlock, 64, 64, 32, 32)
FP8Q_GEMM_KERNEL_FMT(kPairBlockK, 128, 128, 64, 64)
FP8Q_GEMM_KERNEL_FMT(kPairBlockK, 64, 64, 32, 32)
#undef FP8Q_GEMM_KERNEL
#undef FP8Q_GEMM_KERNEL_FMT
#define FP8Q_GEMM_KERNEL_KS2(PAIR, FMT) template __global__ void gemm_kernel<PAIR, 64, 64, 32, 32, false, FMT, 2>(GemmArgs);
FP8Q_GEMM_KERNEL_KS2(kPairTensor, 0)
FP8Q_GEMM_KERNEL_KS2(kPairRow, 0)
FP8Q_GEMM_KERNEL_KS2(kPairBlockE8, 0)
FP8Q_GEMM_KERNEL_KS2(kPairBlock, 0)
FP8Q_GEMM_KERNEL_KS2(kPairBlock, 1)
FP8Q_GEMM_KERNEL_KS2(kPairBlock, 2)
FP8Q_GEMM_KERNEL_KS2(kPairBlock, 3)
FP8Q_GEMM_KERNEL_KS2(kPairBlockK, 0)
FP8Q_GEMM_KERNEL_KS2(kPairBlockK, 1)
FP8Q_GEMM_KERNEL_KS2(kPairBlockK, 2)
FP8Q_GEMM_KERNEL_KS2(kPairBlockK, 3)
#undef FP8Q_GEMM_KERNEL_KS2
#define FP8Q_GEMM_SPLITK(PAIR) template __global__ void gemm_splitk_kernel<PAIR, 128, 128, 32, 64, 0>(GemmArgs);
FP8Q_GEMM_SPLITK(kPairTensor)
FP8Q_GEMM_SPLITK(kPairRow)
FP8Q_GEMM_SPLITK(kPairBlock)
FP8Q_GEMM_SPLITK(kPairBlockK)
#undef FP8Q_GEMM_SPLITK
#define FP8Q_GEMM_THIN_TILES(PAIR, FMT)                                       \
  template __global__ void gemm_thin_kernel<PAIR, 1, 1, false, FMT>(GemmArgs); \
  template __global__ void gemm_thin_kernel<PAIR, 1, 2, false, FMT>(GemmArgs); \
  template __global__ void gemm_thin_kernel<PAIR, 2, 2, false, FMT>(GemmArgs); \
  template __global__ void gemm_thin_kernel<PAIR, 2, 4, false, FMT>(GemmArgs); \
  template __global__ void gemm_thin_kernel<PAIR, 4, 4, false, FMT>(GemmArgs);
FP8Q_GEMM_THIN_TILES(kPairTensor, 0)
FP8Q_GEMM_THIN_TILES(kPairRow, 0)
FP8Q_GEMM_THIN_TILES(kPairBlockE8, 0)
FP8Q_GEMM_THIN_TILES(kPairBlock, 0)
FP8Q_GEMM_THIN_TILES(kPairBlock, 1)
FP8Q_GEMM_THIN_TILES(kPairBlock, 2)
FP8Q_GEMM_THIN_TILES(kPairBlock, 3)
FP8Q_GEMM_THIN_TILES(kPairBlockK, 0)
FP8Q_GEMM_THIN_TILES(kPairBlockK, 1)
FP8Q_GEMM_THIN_TILES(kPairBlockK, 2)
FP8Q_GEMM_THIN_TILES(kPairBlockK, 3)
#undef FP8Q_GEMM_THIN_TILES
template __global__ void gemm_thin_kernel<kPairBlock, 2, 8, true, 0>(GemmArgs);
#define FP8Q_GEMM_GROUPED_THIN(PAIR)                                    \
  template __global__ void gemm_grouped_thin_kernel<PAIR, 1, 1>(GemmGroup); \
  template __global__ void gemm_grouped_thin_kernel<PAIR, 1, 2>(GemmGroup); \
  template __global__ void gemm_grouped_thin_kernel<PAIR, 2, 2>(GemmGroup); \
  template __global__ void gemm_grouped_thin_kernel<PAIR, 2, 4>(GemmGroup); \
  template __global__ void gemm_grouped_thin_kernel<PAIR, 4, 4>(GemmGroup);
FP8Q_GEMM_GROUPED_THIN(kPairTensor)
FP8Q_GEMM_GROUPED_THIN(kPairRow)
FP8Q_GEMM_GROUPED_THIN(kPairBlock)
#undef FP8Q_GEMM_GROUPED_THIN
#define FP8Q_GEMM_LARGE(PAIR, QOUT, FMT) template __global__ void gemm_large_kernel<PAIR, QOUT, FMT>(GemmArgs, int, int);
FP8Q_GEMM_LARGE(kPairTensor, false, 0)
FP8Q_GEMM_LARGE(kPairRow, false, 0)
FP8Q_GEMM_LARGE(kPairBlockE8, false, 0)
FP8Q_GEMM_LARGE(kPairBlock, false, 0)
FP8Q_GEMM_LARGE(kPairBlock, false, 1)
FP8Q_GEMM_LARGE(kPairBlock, false, 2)
FP8Q_GEMM_LARGE(kPairBlock, false, 3)
FP8Q_GEMM_LARGE(kPairBlock, true, 0)
FP8Q_GEMM_LARGE(kPairBlockK, false, 0)
FP8Q_GEMM_LARGE(kPairBlockK, false, 1)
FP8Q_GEMM_LARGE(kPairBlockK, false, 2)
FP8Q_GEMM_LARGE(kPairBlockK, false, 3)
#undef FP8Q_GEMM_LARGE
template __global__ void gemm_kernel<kPairBlock, 128, 128, 64, 64, true, 0>(GemmArgs);
template __global__ void gemm_kernel<kPairBlock, 128, 128, 32, 64, true, 0>(GemmArgs);
template __global__ void gemm_kernel<kPairBlock, 128, 128, 32, 64, true, 0, 1, 2>(GemmArgs);
#define FP8Q_GEMM_GROUPED(PAIR)                                                     \
  template __global__ void gemm_grouped_large_kernel<PAIR>(GemmGroup, int, int);       \
  template __global__ void gemm_grouped_mixed_kernel<PAIR>(GemmGroup, GemmGroup);      \
  template __global__ void gemm_grouped_kernel<PAIR, 128, 128, 64, 64>(GemmGroup);     \
  template __global__ void gemm_grouped_kernel<PAIR, 64, 64, 32, 32>(GemmGroup);       \
  template __global__ void gemm_grouped_kernel<PAIR, 64, 64, 32, 32, 2>(GemmGroup);
FP8Q_GEMM_GROUPED(kPairTensor)
FP8Q_GEMM_GROUPED(kPairRow)
FP8Q_GEMM_GROUPED(kPairBlock)
#undef FP8Q_GEMM_GROUPED

// tile_start of the group for BM x BN tiles; their number, -1 past 2^30 - 1
template <int BM, int BN>
int64_t count_tiles(GemmGroup& gs) {
  int64_t total = 0;
  for (int i = 0; i < gs.count; ++i) {
    gs.tile_start[i] = (int)total;
    total += ((gs.prob[i].M + BM - 1) / BM) * ((gs.prob[i].N + BN - 1) / BN);
    if (total > 0x3fffffff) return -1;
  }
  gs.tile_start[gs.count] = (int)total;
  return total;
}

template <int PAIR, int BM, int BN, int WM, int WN, int KS = 1>
hipError_t launch_grouped_tiles(GemmGroup gs, hipStream_t s) {
  const int64_t total = count_tiles<BM, BN>(gs);
  if (total <= 0) return hipErrorInvalidValue;
  constexpr int threads = (BM / WM) * (BN / WN) * 64 * KS;
  gemm_grouped_kernel<PAIR, BM, BN, WM, WN, KS><<<dim3((unsigned)total), threads, 0, s>>>(gs);
  return hipGetLastError();
}

template <int PAIR>
hipError_t launch_grouped_thin(GemmGroup gs, hipStream_t s) {
  GemmSize sizes[kMaxGroup];
  for (int i = 0; i < gs.count; ++i) sizes[i] = size_of(gs.prob[i]);
  double ns;
  return with_thin(thin_config(sizes, gs.count, ns), [&](auto ti, auto tj) {
    constexpr int TI = decltype(ti)::value, TJ = decltype(tj)::value;
    const int64_t total = count_tiles<TI * 16, TJ * 16>(gs);
    if (total <= 0) return hipErrorInvalidValue;
    gemm_grouped_thin_kernel<PAIR, TI, TJ><<<dim3((unsigned)total), kThinWaves * 64, 0, s>>>(gs);
    return hipGetLastError();
  });
}

template <int PAIR>
hipError_t launch_grouped_large(GemmGroup gs, hipStream_t s) {
  const int64_t total = count_tiles<256, 256>(gs);
  if (total <= 0) return hipErrorInvalidValue;
  const LargePlan p = large_plan(total);
  gemm_grouped_large_kernel<PAIR><<<dim3((unsigned)p.grid), 512, 0, s>>>(gs, p.full, p.parts);
  return hipGetLastError();
}

// The problems with two K groups and the thin ones in one launch, where their
// 64 x 64 tiles together are one round of the CUs; hipErrorNotSupported where
// not.  Two launches of part of the chip each, one after the other, take
// longer (192 tokens, 4096 x (4096 + 256 + 256): 15.4 us, here 11.0).
template <int PAIR>
hipError_t launch_grouped_mixed(GemmGroup grouped, GemmGroup thin, hipStream_t s) {
  const int64_t a = count_tiles<64, 64>(grouped), b = count_tiles<64, 64>(thin);
  if (a <= 0 || b <= 0 || a + b > kCUs) return hipErrorNotSupported;
  gemm_grouped_mixed_kernel<PAIR><<<dim3((unsigned)(a + b)), 512, 0, s>>>(grouped, thin);
  return hipGetLastError();
}

// Each problem goes to the kernel a single call would give it.  The tiled
// kernels without K groups all sum K in one order, so one launch takes every
// problem a single call would give one of them (the tile size from their
// tile count over all: 256 x 256 as takes_large says, 128 x 128 of four waves
// from 256 of them on, else 64 x 64; of a single call's kernels the eight-wave
// one is missing; for a skinny problem among large ones the tile is larger
// than its own, with the same bits); the problems a single call would give
// the thin tiles (which sum in an order of their own, whatever their size) and
// those it would split into K groups go to a second launch, or one each (see
// launch_grouped_mixed).  The thin order is kept where many problems make it
// the slower one: 512 tokens, 8 x (1024 x 1024) 19.9 us, in two K groups 18.7;
// 64 tokens, 3 x (4096 x 4096) 13.1 and 11.6.
template <int PAIR>
hipError_t launch_grouped_pair(const GemmGroup& gs, hipStream_t s) {
  GemmGroup tiled{}, thin{}, grouped{};
  int64_t big = 0, mid = 0, outputs = 0;
  for (int i = 0; i < gs.count; ++i) {
    const GemmArgs& g = gs.prob[i];
    const GemmRoute r = gemm_route(PAIR, size_of(g));
    if (r == kThinTiles) {
      thin.prob[thin.count++] = g;
    } else if (r == kTwoKGroups) {
      grouped.prob[grouped.count++] = g;
    } else {
      tiled.prob[tiled.count++] = g;
      big += tile_count(size_of(g), 256, 256);
      mid += tile_count(size_of(g), 128, 128);
      outputs += g.M * g.N;
    }
  }
  if (tiled.count) {
    const hipError_t e = takes_large(PAIR, big, mid, outputs, gs.prob[0].K) ? launch_grouped_large<PAIR>(tiled, s)
                         : mid >= 256 ? launch_grouped_tiles<PAIR, 128, 128, 64, 64>(tiled, s)
                                      : launch_grouped_tiles<PAIR, 64, 64, 32, 32>(tiled, s);
    if (e != hipSuccess) return e;
  }
  if (thin.count && grouped.count) {
    const hipError_t e = launch_grouped_mixed<PAIR>(grouped, thin, s);
    if (e != hipErrorNotSupported) return e;
  }
  if (thin.count) {
    const hipError_t e = launch_grouped_thin<PAIR>(thin, s);
    if (e != hipSuccess) return e;
  }
  if (grouped.count) return launch_grouped_tiles<PAIR, 64, 64, 32, 32, 2>(grouped, s);
  return hipSuccess;
}

}  // namespace gemm_detail

using namespace gemm_detail;

template <int PAIR>
hipError_t launch_formats(const GemmArgs& g, int formats, hipStream_t s) {
  switch (formats) {
    case 0: return launch_split<PAIR, false, 0>(g, s);
    case 1: return launch_split<PAIR, false, 1>(g, s);
    case 2: return launch_split<PAIR, false, 2>(g, s);
    case 3: return launch_split<PAIR, false, 3>(g, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_gemm(const GemmArgs& g, int pair, int formats, hipStream_t s) {
  if (formats != 0 && pair != kPairBlock && pair != kPairBlockK) return hipErrorInvalidValue;
  switch (pair) {
    case kPairTensor: return launch_split<kPairTensor, false, 0>(g, s);
    case kPairRow: return launch_split<kPairRow, false, 0>(g, s);
    case kPairBlock: return launch_formats<kPairBlock>(g, formats, s);
    case kPairBlockK: return launch_formats<kPairBlockK>(g, formats, s);
    case kPairBlockE8: return launch_split<kPairBlockE8, false, 0>(g, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_gemm_grouped(const GemmGroup& gs, int pair, hipStream_t s) {
  if (gs.count < 1 || gs.count > kMaxGroup) return hipErrorInvalidValue;
  // 32-bit operand offsets inside the kernel: each problem's A, B and C
  // rows span less than 2 GiB
  const int64_t lim = (int64_t)1 << 31;
  for (int i = 0; i < gs.count; ++i) {
    const GemmArgs& g = gs.prob[i];
    if (g.M * g.lda >= lim || g.N * g.ldb >= lim || g.M * 2 * g.ldc >= lim) return hipErrorInvalidValue;
  }
  switch (pair) {
    case kPairTensor: return launch_grouped_pair<kPairTensor>(gs, s);
    case kPairRow: return launch_grouped_pair<kPairRow>(gs, s);
    case kPairBlock: return launch_grouped_pair<kPairBlock>(gs, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_gemm_quantized(const GemmArgs& g, int pair, hipStream_t s) {
  if (pair != kPairBlock || g.N % 128) return hipErrorInvalidValue;
  return launch_split<kPairBlock, true, 0>(g, s);
}

template <int PAIR>
hipError_t launch_splitk_pair(const GemmArgs& g, unsigned grid, hipStream_t s) {
  if (gemm_splitk_route(PAIR, size_of(g), g.splits) == kThinTiles) return launch_thin<PAIR, false, 0>(g, s);
  gemm_splitk_kernel<PAIR, 128, 128, 32, 64, 0><<<dim3(grid), 512, 0, s>>>(g);
  return hipGetLastError();
}

hipError_t launch_gemm_splitk(const GemmArgs& g, int pair, hipStream_t s) {
  if (g.splits <= 1) return launch_gemm(g, pair, 0, s);
  const int64_t tiles = ((g.M + 127) / 128) * ((g.N + 127) / 128);
  if (!g.part || !g.cnt || g.splits > 8 || (g.K / kBK) % g.splits || tiles * g.splits > 256)
    return hipErrorInvalidValue;
  const unsigned grid = (unsigned)(tiles * g.splits);
  switch (pair) {
    case kPairTensor: return launch_splitk_pair<kPairTensor>(g, grid, s);
    case kPairRow: return launch_splitk_pair<kPairRow>(g, grid, s);
    case kPairBlock: return launch_splitk_pair<kPairBlock>(g, grid, s);
    case kPairBlockK: return launch_splitk_pair<kPairBlockK>(g, grid, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace fp8q

// The GemmRoute of an M x N x K problem, for the tests (no part of the ABI):
// `form` is a GemmPair of fp8q_gemm and its relatives, kFormQuantized, or that
// plus one and a GemmPair for fp8q_gemm_splitk.
extern "C" int fp8q_gemm_route(int form, int64_t M, int64_t N, int64_t K) {
  const fp8q::GemmSize s{M, N, K};
  if (form == fp8q::kFormQuantized) return fp8q::gemm_quantized_route(s);
  if (form < fp8q::kFormQuantized) return fp8q::gemm_route(form, s);
  return fp8q::gemm_splitk_route(form - fp8q::kFormQuantized - 1, s, fp8q::gemm_splitk_splits(M, N, K, K, K, N));
}
