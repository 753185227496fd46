// The gated feed-forward block's forward pass on gfx950:
//   H = silu(X Wg^T) * (X Wu^T),  silu(g) = g / (1 + exp(-g)),
// on FP8 operands (X per 1x128 block, both weights per 128x128 block), fp32
// sums, in one kernel: the products of gate and up projection never leave the
// registers unless they are kept for the backward pass.  The kernels are those
// of gemm_tile.h with a tile of B taken half from each weight.
#include "gemm_tile.h"

namespace fp8q {

namespace gemm_detail {

template <int BM, int BN, int WM, int WN, bool QOUT>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void gemm_gated_kernel(GatedArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<kPairBlock, BM, BN, WM, WN>::kBytes];
  int tm, tn;
  tile_coords<BM, BN>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  gemm_tile<kPairBlock, BM, BN, WM, WN, QOUT, 0, 1, false, 1, true>(g, lds, tm, tn);
}

template <int BM, int BN, int WM, int WN, bool QOUT>
hipError_t launch_gated_tiles(const GatedArgs& g, hipStream_t s) {
  const int64_t tiles = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
  gemm_gated_kernel<BM, BN, WM, WN, QOUT><<<dim3((unsigned)tiles), (BM / WM) * (BN / WN) * 64, 0, s>>>(g);
  return hipGetLastError();
}

template <bool QOUT>
hipError_t launch_gated_route(const GatedArgs& g, hipStream_t s) {
  if (((g.M + 255) / 256) * (g.N / 256) >= kCUs) return launch_gated_tiles<256, 256, 128, 64, QOUT>(g, s);
  return launch_gated_tiles<128, 256, 64, 64, QOUT>(g, s);
}

}  // namespace gemm_detail

using namespace gemm_detail;

// The kernels address operands with 32-bit offsets: rows of A that span 2 GiB
// or more are taken in several launches (B is checked by the caller).
hipError_t launch_gemm_gated(const GatedArgs& g, bool quantized, hipStream_t s) {
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
    const hipError_t e = quantized ? launch_gated_route<true>(sub, s) : launch_gated_route<false>(sub, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fp8q
