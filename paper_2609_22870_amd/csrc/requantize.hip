// Activations kept in 8 bits for the backward pass, on gfx950: the codes that a
// forward GEMM took (1x128 units along the features) become the weight-gradient
// GEMM's operand (Eq. 3 in units of 128 tokens, transposed),
//   v = RN32(S code),  S' = RN32(amax over 128 rows of |v| / 448),
//   codes'[c][r] = E4M3 of v / S',
// without the activation ever being held in 16 bits.  A last unit of fewer than
// 128 rows is filled up with zeros, so that the GEMM's contraction stays a whole
// number of units.
//
// Bound by HBM: one byte read and one written an element, and 4 / 128 twice for
// the scales.
#include "ops.h"
#include "quant_tile.h"

namespace fp8q {

namespace quant_detail {

typedef float v2f __attribute__((ext_vector_type(2)));

// Two of the four codes in w (the low or the high 16 bits), as fp32.
template <bool HI>
__device__ __forceinline__ v2f e4m3_values(uint32_t w) {
  return __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HI);
}

__global__ __launch_bounds__(kThreads) void requant_kernel(RequantArgs a, int64_t padded_rows) {
  __shared__ float lds_red[4 * kTile];
  __shared__ uint64_t lds_t[kTile * kTile / 8];
  const int cc = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int64_t tr = blockIdx.y;
  const int64_t r0 = tr * kTile, c0 = (int64_t)blockIdx.x * kTile;
  const int64_t row0 = r0 + rg * 8, c = c0 + cc * 8;

  uint2 w[8];
  float sx[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = row0 + i;
    w[i] = make_uint2(0u, 0u);
    sx[i] = 0.0f;
    if (r < a.rows) {
      w[i] = *reinterpret_cast<const uint2*>(a.codes + r * a.ldc + c);
      sx[i] = a.scales[(int64_t)blockIdx.x * a.rows + r];
    }
  }
  Tile t;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const v2f v0 = e4m3_values<false>(w[i].x), v1 = e4m3_values<true>(w[i].x);
    const v2f v2 = e4m3_values<false>(w[i].y), v3 = e4m3_values<true>(w[i].y);
    t.v[i][0] = v0[0] * sx[i];
    t.v[i][1] = v0[1] * sx[i];
    t.v[i][2] = v1[0] * sx[i];
    t.v[i][3] = v1[1] * sx[i];
    t.v[i][4] = v2[0] * sx[i];
    t.v[i][5] = v2[1] * sx[i];
    t.v[i][6] = v3[0] * sx[i];
    t.v[i][7] = v3[1] * sx[i];
  }

  UnitScale mine;
  float m[8], su[8], ru[8];
  tile_col_max(t, lds_red, m);
  float amax = m[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) amax = (rg & 7) == j ? m[j] : amax;
  share_col_units<false>(amax, a.pow2 != 0, lds_red, mine, su, ru);
  uint32_t packed[8][2];
  encode_patch<kUnitCol, false>(t, su, ru, packed);
  store_patch_transposed(packed, lds_t, a.codes_t, a.ldt, padded_rows, a.cols, r0, c0);
  const int64_t cj = c0 + cc * 8 + rg;
  if (rg < 8) a.scales_t[tr * a.cols + cj] = mine.s;
}

// Gradients of a gated activation H = silu(G) U, from dH and the kept G and U:
//   s = 1 / (1 + exp(-G)),  dG = dH U s (1 + G (1 - s)),  dU = dH G s,
// computed in fp32 and quantized once, as one matrix [dG | dU] of 2 F columns in
// both layouts of the backward GEMMs: codes per 1x128 unit for the data
// gradient's, and transposed codes per 128x1 unit (the rows filled up to a
// multiple of 128 with zeros) for the weight gradient's.  6 bytes read and 4
// written for each element of H; a workgroup holds the 128 x 128 tiles of dG
// and dU at one place in registers.
__device__ __forceinline__ float sigmoid(float g) {
  // exp(-g) from exp2 with the product -g log2(e) in two parts, so that the
  // result keeps fp32 accuracy at any g; past +-88 (where s is 1 or below the
  // normal range) g is held there, which keeps every step finite
  const float x = __builtin_amdgcn_fmed3f(-g, -88.0f, 88.0f);
  constexpr float kLog2e = 0x1.715476p+0f, kLog2eLow = 0x1.4ae0bfp-26f, kLn2 = 0x1.62e430p-1f;
  const float hi = x * kLog2e;
  const float lo = __builtin_fmaf(x, kLog2eLow, __builtin_fmaf(x, kLog2e, -hi));
  const float e = __builtin_amdgcn_exp2f(hi);
  return __builtin_amdgcn_rcpf(1.0f + __builtin_fmaf(e, lo * kLn2, e));
}

// The patch's codes in both layouts.
template <bool E5>
__device__ __forceinline__ void store_dual(const Tile& t, const GatedBackwardArgs& a, float* lds_red, uint64_t* lds_t,
                                           int64_t padded_rows, int64_t tr, int64_t c0) {
  const int cc = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int64_t r0 = tr * kTile, row0 = r0 + rg * 8, c = c0 + cc * 8, cols = 2 * a.F;
  UnitScale mine;
  float su[8], ru[8];
  uint32_t packed[8][2];
  share_row_units<E5>(block_row_amax(t), a.pow2 != 0, mine, su, ru);
  encode_patch<kUnitRow, E5>(t, su, ru, packed);
  store_patch(packed, a.codes_r, a.ldr, a.M, cols, row0, c);
  const int64_t r = row0 + cc;
  if (cc < 8 && r < a.M) a.scales_r[(c >> 7) * a.M + r] = mine.s;
  float m[8];
  tile_col_max(t, lds_red, m);
  float amax = m[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) amax = (rg & 7) == j ? m[j] : amax;
  share_col_units<E5>(amax, a.pow2 != 0, lds_red, mine, su, ru);
  encode_patch<kUnitCol, E5>(t, su, ru, packed);
  store_patch_transposed(packed, lds_t, a.codes_t, a.ldt, padded_rows, cols, r0, c0);
  if (rg < 8) a.scales_t[tr * cols + c0 + cc * 8 + rg] = mine.s;
}

template <bool E5>
__global__ __launch_bounds__(kThreads) void gated_backward_kernel(GatedBackwardArgs a, int64_t padded_rows) {
  __shared__ float lds_red[4 * kTile];
  __shared__ uint64_t lds_t[kTile * kTile / 8];
  const int cc = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int64_t tr = blockIdx.y, c0 = (int64_t)blockIdx.x * kTile;
  const int64_t row0 = tr * kTile + rg * 8, c = c0 + cc * 8;
  Tile dg, du;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = row0 + i;
    uint4 g = make_uint4(0u, 0u, 0u, 0u), u = g, d = g;
    if (r < a.M) {
      g = *reinterpret_cast<const uint4*>(a.pre + r * a.ldp + c);
      u = *reinterpret_cast<const uint4*>(a.pre + r * a.ldp + a.F + c);
      d = *reinterpret_cast<const uint4*>(a.dh + r * a.lddh + c);
    }
    const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, uw[4] = {u.x, u.y, u.z, u.w}, dw[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gv = j & 1 ? bf16_hi(gw[j >> 1]) : bf16_lo(gw[j >> 1]);
      const float uv = j & 1 ? bf16_hi(uw[j >> 1]) : bf16_lo(uw[j >> 1]);
      const float dv = j & 1 ? bf16_hi(dw[j >> 1]) : bf16_lo(dw[j >> 1]);
      const float s = sigmoid(gv);
      dg.v[i][j] = dv * uv * s * __builtin_fmaf(gv, 1.0f - s, 1.0f);
      du.v[i][j] = dv * gv * s;
    }
  }
  store_dual<E5>(dg, a, lds_red, lds_t, padded_rows, tr, c0);
  __syncthreads();  // the tile's LDS is read before the next one's writes
  store_dual<E5>(du, a, lds_red, lds_t, padded_rows, tr, a.F + c0);
}

}  // namespace quant_detail

using namespace quant_detail;

hipError_t launch_requantize_transposed(const RequantArgs& a, hipStream_t s) {
  const int64_t tiles_r = (a.rows + kTile - 1) / kTile;
  const dim3 grid((unsigned)(a.cols / kTile), (unsigned)tiles_r);
  requant_kernel<<<grid, kThreads, 0, s>>>(a, tiles_r * kTile);
  return hipGetLastError();
}

hipError_t launch_gated_backward(const GatedBackwardArgs& a, hipStream_t s) {
  const int64_t tiles_r = (a.M + kTile - 1) / kTile;
  const dim3 grid((unsigned)(a.F / kTile), (unsigned)tiles_r);
  if (a.e5m2)
    gated_backward_kernel<true><<<grid, kThreads, 0, s>>>(a, tiles_r * kTile);
  else
    gated_backward_kernel<false><<<grid, kThreads, 0, s>>>(a, tiles_r * kTile);
  return hipGetLastError();
}

}  // namespace fp8q
