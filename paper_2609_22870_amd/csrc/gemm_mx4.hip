// GEMM of MXFP4 operands on gfx950: E2M1 codes with an E8M0 scale per 32 along K,
//   C[m][n] = sum_k 2^(sA(m, k / 32) - 127) A[m][k] 2^(sB(n, k / 32) - 127) B[n][k],
// fp32 accumulation inside the matrix instruction, which applies the scales, bf16 output.
// The kernels are those of gemm_tile.h: a K step is the 128 bytes that an FP8 step is, but
// 256 codes, two instructions of half an FP8 one's time.
//
// Large products are bound by the way from LDS to the matrix units, then by power: 16384 x 4096 x 12288 385 to
// 415 us, 4.0 to 4.3 PFLOP/s, with the matrix units busy in half of the cycles.  Of 8192^3 the matrix
// instructions alone take 132 us (8.3 PFLOP/s), with the fragments' LDS reads 190, the whole kernel 197 on operands of
// zeros and 240 on normal values: as many cycles, at 1.86 GHz in place of 2.29.  Few rows are bound
// by the bytes that a CU loads, about 85 KB a us: 8 x 4096 x 12288 6.0 us (4.5 TB/s of weights), 64 x
// 17408 x 5120 13.4 (3.7 TB/s).
#include "gemm_tile.h"
#include "rollout.h"

namespace fp8q {

namespace gemm_detail {

template <int TI, int TJ>
__global__ __launch_bounds__(kThinWaves * 64) void gemm_mx4_thin_kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[ThinLds<TI, TJ>::kBytes];
  int tm, tn;
  tile_coords<TI * 16, TJ * 16>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  thin_tile<kPairMx4, TI, TJ, false, 0>(g, lds, tm, tn);
}

template <int BM, int BN, int WM, int WN, int KS = 1>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64 * KS) void gemm_mx4_kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<kPairMx4, BM, BN, WM, WN, KS>::kBytes];
  int tm, tn;
  tile_coords<BM, BN>(g.M, g.N, g.K, blockIdx.x, tm, tn);
  gemm_tile<kPairMx4, BM, BN, WM, WN, false, 0, KS>(g, lds, tm, tn);
}

// 256 x 256 tiles, the last round cut as gemm.hip's large_tiles cuts it.
__global__ __launch_bounds__(512) void gemm_mx4_large_kernel(GemmArgs g, int full, int parts) {
  constexpr int kWhole = TileLds<kPairMx4, 256, 256, 128, 64>::kBytes,
                kHalf = TileLds<kPairMx4, 128, 256, 64, 64>::kBytes,
                kQuarter = TileLds<kPairMx4, 128, 128, 32, 64>::kBytes;
  constexpr int kMost = kWhole > kHalf ? kWhole : kHalf;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kMost > kQuarter ? kMost : kQuarter];
  const int b = blockIdx.x;
  int tm, tn;
  if (b < full) {
    raster<256, 256>(g.M, g.N, g.K, xcd_order(full, b), tm, tn);
    gemm_tile<kPairMx4, 256, 256, 128, 64, false, 0>(g, lds, tm, tn);
    return;
  }
  const int t = xcd_order((int)gridDim.x - full, b - full);  // (full % 8 == 0: the XCD is still b % 8)
  const int part = t & (parts - 1);
  raster<256, 256>(g.M, g.N, g.K, full + (parts == 4 ? t >> 2 : t >> 1), tm, tn);
  tm = 2 * tm + (part & 1);
  if ((int64_t)tm * 128 >= g.M) return;  // (the whole workgroup: a part past the edge of C)
  if (parts == 4) {
    tn = 2 * tn + (part >> 1);
    if ((int64_t)tn * 128 >= g.N) return;
    gemm_tile<kPairMx4, 128, 128, 32, 64, false, 0>(g, lds, tm, tn);
  } else {
    gemm_tile<kPairMx4, 128, 256, 64, 64, false, 0>(g, lds, tm, tn);
  }
}

namespace {

// The kernel of a product of K bytes a row: that of FP8 codes with power-of-two scales, whose
// steps of 128 bytes of a row these are, but for two kinds of sizes where half an
// instruction's time shows: large tiles also where they fill whole rounds of the CUs (4096 x 512 x 4096 12.2
// us, 128 x 128 tiles 13.5; 16384 x 512 x 12288 116 and 123), and up to two 64 x 64 tiles a CU before
// 128 x 128 tiles of eight waves, but for a single row of them (512 x 4096 x 4096 9.1 us, eight waves
// 11.8; 512 x 12288 x 4096 27.8 and 31.1; 192 x 1024 x 8192 4.9 and 5.8; 64 x 5120 x 17408 23.1 and 21.1).
// Over 110 sizes, half of them random, the choice is about 1% above the best of these kernels.
inline GemmRoute mx4_route(const GemmSize& s) {
  const GemmRoute r = gemm_route(kPairBlockE8, s);
  if (r == kMidTiles && tile_count(s, 256, 256) % kCUs == 0) return kLargeTiles;
  if (r == kEightWaves && s.M > 64 && tile_count(s, 64, 64) <= 2 * kCUs) return kSmallTiles;
  return r;
}

// Thin tiles of three strips of 16 columns in place of four where all of them have a CU each: a CU
// then loads 80 or 112 rows of K in place of 96 or 128, which is what these products wait for
// (64 x 17408 x 5120 20.4 us with 32 x 64 tiles, 17.6 with 32 x 48; 64 x 25600 x 5120 28.4 and 24.5;
// 128 x 25600 x 5120 35.5 with 64 x 64, 31.1 with 64 x 48, weights from memory.  28 of 510 random sizes: 7%
// faster on average, at most 2% slower).
inline bool three_strips(const GemmSize& s, int config) {
  return (config == kThin32x64 || config == kThin64x64) && tile_count(s, kThinM[config], 48) <= kCUs;
}

template <int BM, int BN, int WM, int WN, int KS = 1>
hipError_t launch_mx4_tiles(const GemmArgs& g, hipStream_t s) {
  const int64_t tiles = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
  gemm_mx4_kernel<BM, BN, WM, WN, KS><<<dim3((unsigned)tiles), (BM / WM) * (BN / WN) * 64 * KS, 0, s>>>(g);
  return hipGetLastError();
}

template <int TI, int TJ>
hipError_t launch_mx4_thin(const GemmArgs& g, hipStream_t s) {
  const int64_t tiles = ((g.M + TI * 16 - 1) / (TI * 16)) * ((g.N + TJ * 16 - 1) / (TJ * 16));
  if (tiles <= 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
  gemm_mx4_thin_kernel<TI, TJ><<<dim3((unsigned)tiles), kThinWaves * 64, 0, s>>>(g);
  return hipGetLastError();
}

// A problem whose operands and output span less than 2 GiB each.
hipError_t launch_mx4_sub(const GemmArgs& g, hipStream_t s) {
  const GemmSize size{g.M, g.N, g.K};
  switch (mx4_route(size)) {
    case kLargeTiles: {
      const int64_t tiles = tile_count(size, 256, 256);
      if (tiles <= 0 || tiles > 0x3fffffff) return hipErrorInvalidValue;
      const LargePlan p = large_plan(tiles);
      gemm_mx4_large_kernel<<<dim3((unsigned)p.grid), 512, 0, s>>>(g, p.full, p.parts);
      return hipGetLastError();
    }
    case kMidTiles: return launch_mx4_tiles<128, 128, 64, 64>(g, s);
    case kEightWaves: return launch_mx4_tiles<128, 128, 32, 64>(g, s);
    case kSmallTiles: return launch_mx4_tiles<64, 64, 32, 32>(g, s);
    case kTwoKGroups: return launch_mx4_tiles<64, 64, 32, 32, 2>(g, s);
    case kThinTiles: {
      double ns;
      const int config = thin_config(&size, 1, ns);
      if (three_strips(size, config)) return config == kThin32x64 ? launch_mx4_thin<2, 3>(g, s) : launch_mx4_thin<4, 3>(g, s);
      switch (config) {
        case kThin16x16: return launch_mx4_thin<1, 1>(g, s);
        case kThin16x32: return launch_mx4_thin<1, 2>(g, s);
        case kThin32x32: return launch_mx4_thin<2, 2>(g, s);
        case kThin32x64: return launch_mx4_thin<2, 4>(g, s);
        case kThin64x64: return launch_mx4_thin<4, 4>(g, s);
        default: break;
      }
      break;
    }
    default: break;
  }
  return hipErrorInvalidValue;
}

}  // namespace

}  // namespace gemm_detail

hipError_t launch_gemm_mx4(const GemmArgs& g, hipStream_t s) {
  // the kernels' 32-bit offsets: rows of A, B and C that span less than 2 GiB a launch
  const int64_t lim = (int64_t)1 << 31;
  int64_t mstep = g.M, nstep = g.N;
  if (g.M * g.lda >= lim) mstep = (lim - 1) / g.lda / 256 * 256;
  if (g.M * 2 * g.ldc >= lim) {
    const int64_t c = (lim - 1) / (2 * g.ldc) / 256 * 256;
    mstep = c < mstep ? c : mstep;
  }
  // (whole pairs of the 1024-column bands that walk K in two directions)
  if (g.N * g.ldb >= lim) nstep = (lim - 1) / g.ldb / 2048 * 2048;
  if (mstep <= 0 || nstep <= 0) return hipErrorInvalidValue;
  for (int64_t m = 0; m < g.M; m += mstep) {
    for (int64_t n = 0; n < g.N; n += nstep) {
      GemmArgs sub = g;
      sub.M = g.M - m < mstep ? g.M - m : mstep;
      sub.N = g.N - n < nstep ? g.N - n : nstep;
      sub.A = g.A + m * g.lda;
      sub.B = g.B + n * g.ldb;
      sub.C = g.C + m * g.ldc + n;
      // (the scales keep the whole problem's strides)
      sub.sA = g.sA + 2 * m;
      sub.sB = g.sB + 2 * n;
      sub.sa_count = g.sa_count - 2 * m;
      sub.sb_count = g.sb_count - 2 * n;
      const hipError_t e = gemm_detail::launch_mx4_sub(sub, s);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace fp8q

// The GemmRoute of a product of K codes (a multiple of 256), for the tests (no part of the ABI).
extern "C" int fp8q_gemm_mx4_route(int64_t M, int64_t N, int64_t K) {
  return fp8q::gemm_detail::mx4_route(fp8q::GemmSize{M, N, K / 2});
}
