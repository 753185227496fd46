// The gated feed-forward block's forward pass on gfx950:
//   H = silu(X Wg^T) * (X Wu^T),  silu(g) = g / (1 + exp(-g)),
// on FP8 operands (X per 1x128 block, both weights per 128x128 block), fp32
// sums, in one kernel: the products of gate and up projection never leave the
// registers unless they are kept for the backward pass.  The kernels are those
// of gemm_tile.h with a tile of B taken half from each weight.  Bound by the matrix
// cores and the promotion beside it, as the plain GEMM: 16384 x 4096 x 12288 with
// quantized output and kept pre-activations 1.51 ms (2.2 PFLOP/s); 8 tokens by the
// weights, 18.2 us with them in memory (5.5 TB/s; 16.3 with them in the last-level cache).
#include "gemm_tile.h"

namespace fp8q {

namespace gemm_detail {

template <int BM, int BN, int WM, int WN, bool QOUT, int KS = 1>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64 * KS) void gemm_gated_kernel(GatedArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<kPairBlock, BM, BN, WM, WN, KS>::kBytes];
  int tm, tn;
  tile_coords<BM, BN>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  gemm_tile<kPairBlock, BM, BN, WM, WN, QOUT, 0, KS, false, 1, true>(g, lds, tm, tn);
}

template <int TI, int TJ>
__global__ __launch_bounds__(kThinWaves * 64) void gemm_gated_thin_kernel(GatedArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[ThinLds<TI, TJ>::kBytes];
  int tm, tn;
  tile_coords<TI * 16, TJ * 16>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  thin_tile<kPairBlock, TI, TJ, false, 0, true>(g, lds, tm, tn);
}

// 256 x 256 tiles with the last round cut as gemm.hip's large_tiles cuts it: the
// tiles past `full` in `parts` each, 2 of 128 x 256 or 4 of 128 x 128 (the latter
// not with quantized output, whose units are two of their tiles wide).
template <bool QOUT>
__global__ __launch_bounds__(512) void gemm_gated_large_kernel(GatedArgs g, int full, int parts) {
  constexpr int kWhole = TileLds<kPairBlock, 256, 256, 128, 64>::kBytes,
                kHalf = TileLds<kPairBlock, 128, 256, 64, 64>::kBytes,
                kQuarter = TileLds<kPairBlock, 128, 128, 32, 64>::kBytes;
  constexpr int kMost = kWhole > kHalf ? kWhole : kHalf;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kMost > kQuarter ? kMost : kQuarter];
  const int b = blockIdx.x;
  int tm, tn;
  if (b < full) {
    raster<256, 256>(g.M, g.N, g.K, xcd_order(full, b), tm, tn);
    gemm_tile<kPairBlock, 256, 256, 128, 64, QOUT, 0, 1, false, 1, true>(g, lds, tm, tn);
    return;
  }
  const int t = xcd_order((int)gridDim.x - full, b - full);  // (full % 8 == 0: the XCD is still b % 8)
  const int part = t & (parts - 1);
  raster<256, 256>(g.M, g.N, g.K, full + (parts == 4 ? t >> 2 : t >> 1), tm, tn);
  tm = 2 * tm + (part & 1);
  if ((int64_t)tm * 128 >= g.M) return;  // (the whole workgroup: a part past the edge of H)
  if constexpr (!QOUT) {
    if (parts == 4) {
      gemm_tile<kPairBlock, 128, 128, 32, 64, false, 0, 1, false, 1, true>(g, lds, tm, 2 * tn + (part >> 1));
      return;
    }
  }
  gemm_tile<kPairBlock, 128, 256, 64, 64, QOUT, 0, 1, false, 1, true>(g, lds, tm, tn);
}

template <bool QOUT>
hipError_t launch_gated_large(const GatedArgs& g, hipStream_t s) {
  const int64_t tiles = tile_count(GemmSize{g.M, g.N, g.K}, 256, 256);
  if (tiles <= 0 || tiles > 0x3fffffff) return hipErrorInvalidValue;
  LargePlan p = large_plan(tiles);
  if (QOUT && p.parts == 4) {
    p.parts = 2;
    p.grid = p.full + 2 * (int)(tiles - p.full);
  }
  gemm_gated_large_kernel<QOUT><<<dim3((unsigned)p.grid), 512, 0, s>>>(g, p.full, p.parts);
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, bool QOUT, int KS = 1>
hipError_t launch_gated_tiles(const GatedArgs& g, hipStream_t s) {
  const int64_t tiles = tile_count(GemmSize{g.M, g.N, g.K}, BM, BN);
  if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
  gemm_gated_kernel<BM, BN, WM, WN, QOUT, KS><<<dim3((unsigned)tiles), (BM / WM) * (BN / WN) * 64 * KS, 0, s>>>(g);
  return hipGetLastError();
}

template <int TI, int TJ>
hipError_t launch_gated_thin(const GatedArgs& g, hipStream_t s) {
  const int64_t tiles = tile_count(GemmSize{g.M, g.N, g.K}, TI * 16, TJ * 16);
  if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
  gemm_gated_thin_kernel<TI, TJ><<<dim3((unsigned)tiles), kThinWaves * 64, 0, s>>>(g);
  return hipGetLastError();
}

// One launch, by the route of the whole problem `size` (g may be a part of it).
hipError_t launch_gated_route(const GatedArgs& g, const GemmSize& size, bool quantized, hipStream_t s) {
  const int route = gated_route(size);
  if (quantized) {
    if (gated_through_bf16(size)) return hipErrorInvalidValue;
    return route == kLargeTiles ? launch_gated_large<true>(g, s) : launch_gated_tiles<128, 256, 64, 64, true>(g, s);
  }
  switch (route) {
    case kLargeTiles: return launch_gated_large<false>(g, s);
    case kHalfTiles: return launch_gated_tiles<128, 256, 64, 64, false>(g, s);
    case kMidTiles: return launch_gated_tiles<128, 128, 64, 64, false>(g, s);
    case kEightWaves: return launch_gated_tiles<128, 128, 32, 64, false>(g, s);
    case kSmallTiles: return launch_gated_tiles<64, 64, 32, 32, false>(g, s);
    case kTwoKGroups: return launch_gated_tiles<64, 64, 32, 32, false, 2>(g, s);
    case kThinTiles:
      switch (gated_thin_config(size)) {
        case kThin16x32: return launch_gated_thin<1, 2>(g, s);
        case kThin32x32: return launch_gated_thin<2, 2>(g, s);
        case kThin32x64: return launch_gated_thin<2, 4>(g, s);
        case kThin64x64: return launch_gated_thin<4, 4>(g, s);
        default: return hipErrorInvalidValue;
      }
    default: return hipErrorInvalidValue;
  }
}

// The kernels address operands with 32-bit offsets: rows of A that span 2 GiB
// or more are taken in several launches (B is checked by the caller).
hipError_t launch_parts(const GatedArgs& g, bool quantized, hipStream_t s) {
  const int64_t lim = (int64_t)1 << 31;
  if (g.N % 256 || g.N * g.ldb >= lim) return hipErrorInvalidValue;
  int64_t step = g.M;
  if (g.M * g.lda >= lim) step = ((lim - 1) / g.lda) / 256 * 256;
  if (step > ((int64_t)1 << 28)) step = (int64_t)1 << 28;
  if (step <= 0) return hipErrorInvalidValue;
  for (int64_t m = 0; m < g.M; m += step) {
    GatedArgs sub = g;
    sub.M = g.M - m < step ? g.M - m : step;
    sub.A = g.A + m * g.lda;
    sub.sA = g.sA + m;
    sub.sa_count = g.sa_count - m;
    if (g.pre) sub.pre = g.pre + m * g.ldp;
    if (quantized) {
      sub.Cq = g.Cq + m * g.ldq;
      sub.Cs = g.Cs + m;
    } else {
      sub.C = g.C + m * g.ldc;
    }
    const hipError_t e = launch_gated_route(sub, GemmSize{g.M, g.N, g.K}, quantized, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace gemm_detail

using namespace gemm_detail;

bool gated_needs_bf16(int64_t M, int64_t F, int64_t K) { return gated_through_bf16(GemmSize{M, 2 * F, K}); }

hipError_t launch_gemm_gated(const GatedArgs& g, bool quantized, hipStream_t s) {
  if (!quantized || !gated_through_bf16(GemmSize{g.M, g.N, g.K})) return launch_parts(g, quantized, s);
  if (!g.C) return hipErrorInvalidValue;
  const hipError_t e = launch_parts(g, false, s);
  if (e != hipSuccess) return e;
  QuantArgs q{};
  q.x = g.C;
  q.rows = g.M;
  q.cols = g.N / 2;
  q.ldx = g.ldc;
  q.codes = g.Cq;
  q.ldc = g.ldq;
  q.scales = g.Cs;
  return launch_quantize(q, FP8Q_BLOCK_1x128, false, g.M * (g.N / 256), s);
}

}  // namespace fp8q

// The route of a gated product, for the tests (no part of the ABI): a GemmRoute
// or kHalfTiles, plus 10 times the thin tile, plus 100 where quantized output goes
// through bf16.
extern "C" int fp8q_gated_route(int64_t M, int64_t F, int64_t K) {
  const fp8q::GemmSize s{M, 2 * F, K};
  const int r = fp8q::gated_route(s);
  return r + (r == fp8q::kThinTiles ? 10 * fp8q::gated_thin_config(s) : 0) + (fp8q::gated_through_bf16(s) ? 100 : 0);
}
