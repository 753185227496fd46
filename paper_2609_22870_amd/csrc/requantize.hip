// Operands of the backward GEMMs that are made from what the forward pass kept,
// on gfx950: a weight gradient's from an activation's 8-bit codes, and the two
// of a gated activation's gradient.
//
// A workgroup takes a tile of 128 x 128 elements, 8 rows x COLS columns a thread
// in fp32 registers.  The 128 / COLS lanes of a tile row share its 1x128 unit;
// the rows' groups meet in LDS for the 128x1 units' maxima.  Every lane forms the
// scales it needs itself (code_scale: ten instructions, less than the
// shuffles or LDS exchanges and barriers of handing them round).  Codes that leave
// transposed are packed along the rows, so that a thread's conversions already
// give eight tokens of one column, and go through LDS only to leave in 16-byte
// pieces.
#include "device_common.h"
#include "ops.h"

namespace fp8q {

namespace requant_detail {

constexpr int kTile = 128;

typedef float v2f __attribute__((ext_vector_type(2)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));

template <int COLS>
struct Patch {
  float v[8][COLS];
};

// Threads of a tile, lanes of a tile row, and groups of eight rows of a wave.
template <int COLS>
struct Shape {
  static constexpr int kLanes = kTile / COLS, kThreads = kLanes * kTile / 8, kWaves = kThreads / 64;
  static constexpr int kGroups = 64 / kLanes;
};

// Four codes of the quotients by one unit's scale.
template <bool E5>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, const CodeScale& u) {
  auto q = [&](float x) { return fast_quotient(x, u.d, u.r); };
  return code_pack2<E5, true>(q(c), q(d), code_pack2<E5, false>(q(a), q(b), 0u));
}

// Workgroup b's tile, tiles numbered along the columns first.  Workgroup b runs on
// XCD b % 8; each XCD takes a range of consecutive tiles, so that its L2 sees
// whole runs of each row (16384 x 12288 requantized 98.1 us in grid order, 88.3
// so).
__device__ __forceinline__ void tile_of(int tiles_c, int& tr, int& tc) {
  const int total = gridDim.x, b = blockIdx.x, xcd = b & 7, per = total >> 3, extra = total & 7;
  const int t = xcd * per + (xcd < extra ? xcd : extra) + (b >> 3);
  tr = t / tiles_c;
  tc = t - tr * tiles_c;
}

// Maximum over the lanes of a tile row.
template <int COLS>
__device__ __forceinline__ float row_max(float v) {
  v = row16_magnitude_max(v);
  return Shape<COLS>::kLanes > 16 ? magnitude_max(with_lane16(v)) : v;
}

// The patch's 1x128 codes to rows row0 .. row0 + 7 (those below `rows`) from
// column c on, and their scales, [cols / 128][rows] at block c / 128.
template <int COLS, bool E5>
__device__ __forceinline__ void store_rows(const Patch<COLS>& p, bool pow2, int64_t row0, int64_t rows, int64_t c,
                                           uint8_t* codes, int64_t ldc, float* scales) {
  const int cc = threadIdx.x % Shape<COLS>::kLanes;
  uint8_t* const to = codes + row0 * ldc + c;  // (row i: a scalar further on)
  float* const st = scales + (c >> 7) * rows + row0;
  const int left = (int)(rows - row0 < 8 ? rows - row0 : 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < COLS; ++j) m = fmaxf(m, fabsf(p.v[i][j]));
    const CodeScale u = code_scale<E5>(row_max<COLS>(m), pow2);
    const bool lifted = __any(u.lift != 1.0f);
    uint32_t w[COLS / 4];
#pragma unroll
    for (int j = 0; j < COLS; j += 4) {
      float v[4] = {p.v[i][j], p.v[i][j + 1], p.v[i][j + 2], p.v[i][j + 3]};
      if (lifted) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = lifted_value<E5>(v[e], u);
      }
      w[j / 4] = codes4<E5>(v[0], v[1], v[2], v[3], u);
    }
    if (i < left) {
      if constexpr (COLS == 8)
        *reinterpret_cast<uint2*>(to + i * ldc) = make_uint2(w[0], w[1]);
      else
        *reinterpret_cast<uint32_t*>(to + i * ldc) = w[0];
      if (cc == 0) st[i] = u.s;
    }
  }
}

// Column maxima of the wave's rows, to lds[wave][128].
template <int COLS>
__device__ __forceinline__ void leave_col_max(const Patch<COLS>& p, float (*lds)[kTile]) {
  constexpr int L = Shape<COLS>::kLanes;
  const int cc = threadIdx.x % L, lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < COLS; ++j) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(p.v[i][j]));
    if constexpr (L == 16) m = magnitude_max(with_lane16(m));
    m = magnitude_max(with_lane32(m));
    if (lane < L) lds[threadIdx.x >> 6][cc * COLS + j] = m;
  }
}

// The patch's 128x1 codes, transposed, to LDS: line j of the tile (128 bytes, a
// column's 128 tokens) holds in its eight-byte chunk g ^ (j / COLS % 16) the
// tokens of row group g.  Then the scales, at scales + the tile's first column.
template <int COLS, bool E5>
__device__ __forceinline__ void leave_columns(const Patch<COLS>& p, bool pow2, const float (*lds)[kTile],
                                              uint64_t* lines, float* scales) {
  constexpr int L = Shape<COLS>::kLanes, W = Shape<COLS>::kWaves;
  const int cc = threadIdx.x % L, rg = threadIdx.x / L;
#pragma unroll
  for (int j = 0; j < COLS; ++j) {
    float m = lds[0][cc * COLS + j];
#pragma unroll
    for (int w = 1; w < W; ++w) m = magnitude_max(make_float2(m, lds[w][cc * COLS + j]));
    const CodeScale u = code_scale<E5>(m, pow2);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p.v[i][j];
    if (__any(u.lift != 1.0f)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = lifted_value<E5>(v[i], u);
    }
    const uint32_t w[2] = {codes4<E5>(v[0], v[1], v[2], v[3], u), codes4<E5>(v[4], v[5], v[6], v[7], u)};
    lines[(cc * COLS + j) * 16 + (rg ^ (cc & 15))] = (uint64_t)w[0] | ((uint64_t)w[1] << 32);
    if (rg == 0) scales[cc * COLS + j] = u.s;
  }
}

// The tile's lines from LDS to codes_t[c0 + j][r0 ..], in 16-byte pieces.
template <int COLS>
__device__ __forceinline__ void store_lines(const uint64_t* lines, uint8_t* codes_t, int64_t ldt, int64_t c0,
                                            int64_t r0) {
  constexpr int T = Shape<COLS>::kThreads;
#pragma unroll
  for (int x = threadIdx.x; x < kTile * 8; x += T) {
    const int j = x >> 3, q = x & 7, sw = (j / COLS) & 15;
    const uint64_t a = lines[j * 16 + ((2 * q) ^ sw)], b = lines[j * 16 + ((2 * q + 1) ^ sw)];
    *reinterpret_cast<uint4*>(codes_t + (c0 + j) * ldt + r0 + q * 16) =
        make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32));
  }
}

// Eight bytes that nothing reads again: they go past the caches, which keep what
// is about to be read (4096 x 5120 gated gradient 62 -> 56 us).
__device__ __forceinline__ uint2 read_once(const void* p) {
  const v2u v = __builtin_nontemporal_load(static_cast<const v2u*>(p));
  return make_uint2(v[0], v[1]);
}

// Two of the four codes in w (the low or the high 16 bits), as fp32.
template <bool HI>
__device__ __forceinline__ v2f e4m3_values(uint32_t w) {
  return __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HI);
}

// Activations kept in 8 bits: the codes that a forward GEMM took (1x128 units
// along the features) become the weight-gradient GEMM's operand (Eq. 3 in units
// of 128 tokens, transposed),
//   v = RN32(S code),  S' = RN32(amax over 128 rows of |v| / 448),
//   codes'[c][r] = E4M3 of v / S',
// without the activation ever being held in 16 bits.  A last unit of fewer than
// 128 rows is filled up with zeros, so that the GEMM's contraction stays a whole
// number of units.  Bound by HBM: one byte read and one written an element, and
// 4 / 128 twice for the scales (16384 x 12288 84 us, 4.9 TB/s).
constexpr int kRequantCols = 8;

__global__ __launch_bounds__(Shape<kRequantCols>::kThreads) void requant_kernel(RequantArgs a) {
  constexpr int C = kRequantCols, L = Shape<C>::kLanes;
  __shared__ float lds[Shape<C>::kWaves][kTile];
  __shared__ uint64_t lines[kTile * kTile / 8];
  const int cc = threadIdx.x % L, rg = threadIdx.x / L;
  int tr, tc;
  tile_of((int)(a.cols / kTile), tr, tc);
  const int64_t r0 = (int64_t)tr * kTile, c0 = (int64_t)tc * kTile;
  const int64_t row0 = r0 + rg * 8, c = c0 + cc * C;
  uint2 w[8];
  float s[8];
  const uint8_t* const pc = a.codes + row0 * a.ldc + c;
  const float* const ps = a.scales + (int64_t)tc * a.rows + row0;
  const int left = (int)(a.rows - row0 < 8 ? a.rows - row0 : 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[i] = make_uint2(0u, 0u);
    s[i] = 0.0f;
    if (i < left) {
      w[i] = *reinterpret_cast<const uint2*>(pc + i * a.ldc);
      s[i] = ps[i];
    }
  }
  Patch<C> p;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const v2f v[4] = {e4m3_values<false>(w[i].x), e4m3_values<true>(w[i].x), e4m3_values<false>(w[i].y),
                      e4m3_values<true>(w[i].y)};
#pragma unroll
    for (int j = 0; j < C; ++j) p.v[i][j] = v[j >> 1][j & 1] * s[i];
  }
  leave_col_max<C>(p, lds);
  __syncthreads();
  leave_columns<C, false>(p, a.pow2 != 0, lds, lines, a.scales_t + tr * a.cols + c0);
  __syncthreads();
  store_lines<C>(lines, a.codes_t, a.ldt, c0, r0);
}

// Gradients of a gated activation H = silu(G) U, from dH and the kept G and U:
//   s = 1 / (1 + exp(-G)),  dG = dH U s (1 + G (1 - s)),  dU = dH G s,
// computed in fp32 and quantized once, as one matrix [dG | dU] of 2 F columns in
// both layouts of the backward GEMMs: codes per 1x128 unit for the data
// gradient's, and transposed codes per 128x1 unit (the rows filled up to a
// multiple of 128 with zeros) for the weight gradient's.  6 bytes read and 4
// written for each element of H (16384 x 12288 430 us, 4.7 TB/s).  A workgroup holds the tiles of dG and dU at
// one place: 8 x 4 patches, so that both fit the registers of four waves per
// SIMD.  log2(e) is kLog2e, sixteen bits whose product with a bf16 G is exact, and a
// rest of which kRest is ln 2 times: exp(-G) = 2^(-G kLog2e) (1 - G kRest), good to fp32 (at
// |G| = 87 the next term is 2^-23), and overflows to s = 0 as it should.  (One rounded
// product was off by |G| 2^-24 of the value.)
constexpr float kLog2e = 0x1.7154p+0f, kRest = 0x1.480fb6p-18f;
constexpr int kGatedCols = 4;

template <bool E5>
__global__ __launch_bounds__(Shape<kGatedCols>::kThreads) void gated_backward_kernel(GatedBackwardArgs a) {
  constexpr int C = kGatedCols, L = Shape<C>::kLanes;
  __shared__ float lds[2][Shape<C>::kWaves][kTile];
  __shared__ uint64_t lines[2][kTile * kTile / 8];
  const int cc = threadIdx.x % L, rg = threadIdx.x / L;
  int tr, tc;
  tile_of((int)(a.F / kTile), tr, tc);
  const int64_t r0 = (int64_t)tr * kTile, c0 = (int64_t)tc * kTile;
  const int64_t row0 = r0 + rg * 8, c = c0 + cc * C;
  uint2 g[8], u[8], d[8];
  const uint16_t *const pg = a.pre + row0 * a.ldp + c, *const pu = pg + a.F, *const pd = a.dh + row0 * a.lddh + c;
  const int left = (int)(a.M - row0 < 8 ? a.M - row0 : 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    g[i] = u[i] = d[i] = make_uint2(0u, 0u);
    if (i < left) {
      g[i] = read_once(pg + i * a.ldp);
      u[i] = read_once(pu + i * a.ldp);
      d[i] = read_once(pd + i * a.lddh);
    }
  }
  Patch<C> dg, du;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t gw[2] = {g[i].x, g[i].y}, uw[2] = {u[i].x, u[i].y}, dw[2] = {d[i].x, d[i].y};
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const float gv = j & 1 ? bf16_hi(gw[j >> 1]) : bf16_lo(gw[j >> 1]);
      const float uv = j & 1 ? bf16_hi(uw[j >> 1]) : bf16_lo(uw[j >> 1]);
      const float dv = j & 1 ? bf16_hi(dw[j >> 1]) : bf16_lo(dw[j >> 1]);
      const float e = __builtin_amdgcn_exp2f(gv * -kLog2e) * __builtin_fmaf(gv, -kRest, 1.0f);
      const float s = __builtin_amdgcn_rcpf(1.0f + e);
      const float ds = dv * s, dgs = ds * gv;
      dg.v[i][j] = uv * __builtin_fmaf(dgs, 1.0f - s, ds);
      du.v[i][j] = dgs;
    }
  }
  const bool pow2 = a.pow2 != 0;
  leave_col_max<C>(dg, lds[0]);
  leave_col_max<C>(du, lds[1]);
  store_rows<C, E5>(dg, pow2, row0, a.M, c, a.codes_r, a.ldr, a.scales_r);
  store_rows<C, E5>(du, pow2, row0, a.M, a.F + c, a.codes_r, a.ldr, a.scales_r);
  __syncthreads();
  float* const st = a.scales_t + tr * 2 * a.F + c0;
  leave_columns<C, E5>(dg, pow2, lds[0], lines[0], st);
  leave_columns<C, E5>(du, pow2, lds[1], lines[1], st + a.F);
  __syncthreads();
  store_lines<C>(lines[0], a.codes_t, a.ldt, c0, r0);
  store_lines<C>(lines[1], a.codes_t, a.ldt, a.F + c0, r0);
}

}  // namespace requant_detail

using namespace requant_detail;

hipError_t launch_requantize_transposed(const RequantArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.cols / kTile * ((a.rows + kTile - 1) / kTile)));
  requant_kernel<<<grid, Shape<kRequantCols>::kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_gated_backward(const GatedBackwardArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.F / kTile * ((a.M + kTile - 1) / kTile)));
  if (a.e5m2)
    gated_backward_kernel<true><<<grid, Shape<kGatedCols>::kThreads, 0, s>>>(a);
  else
    gated_backward_kernel<false><<<grid, Shape<kGatedCols>::kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace fp8q
