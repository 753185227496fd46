// The 128 x 128 tile of the quantizers on gfx950: a workgroup of 256 threads
// holds it in 8 x 8 patches, takes its units' maxima and scales, and writes its
// codes plain or transposed.
#pragma once

#include "device_common.h"
#include "internal.h"

namespace fp8q {

namespace quant_detail {

constexpr int kTile = 128;
constexpr int kThreads = 256;

struct Tile {
  float v[8][8];  // [row i][column j] of this thread's 8 x 8 patch
};

// Rows row0 .. row0+7, columns c .. c+7 of x (zeros outside).
__device__ __forceinline__ void load_patch(const QuantArgs& a, int64_t row0, int64_t c, Tile& t) {
  const bool col_ok = c < a.cols;
  uint4 w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = row0 + i;
    w[i] = make_uint4(0u, 0u, 0u, 0u);
    if (col_ok && r < a.rows) w[i] = *reinterpret_cast<const uint4*>(a.x + r * a.ldx + c);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    t.v[i][0] = bf16_lo(w[i].x);
    t.v[i][1] = bf16_hi(w[i].x);
    t.v[i][2] = bf16_lo(w[i].y);
    t.v[i][3] = bf16_hi(w[i].y);
    t.v[i][4] = bf16_lo(w[i].z);
    t.v[i][5] = bf16_hi(w[i].z);
    t.v[i][6] = bf16_lo(w[i].w);
    t.v[i][7] = bf16_hi(w[i].w);
  }
}

__device__ __forceinline__ float row_partial_max(const Tile& t, int i) {
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(t.v[i][j]));
  return m;
}

__device__ __forceinline__ float col_partial_max(const Tile& t, int j) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(t.v[i][j]));
  return m;
}

// Column maxima over the whole 128-row tile: eight per thread (its columns).
__device__ __forceinline__ void tile_col_max(const Tile& t, float* lds_cols /*[4][128]*/, float out[8]) {
  const int cc = threadIdx.x & 15, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float m = across_rows_max(col_partial_max(t, j));
    if (lane < 16) lds_cols[wave * kTile + cc * 8 + j] = m;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int col = cc * 8 + j;
    out[j] = fmaxf(fmaxf(lds_cols[col], lds_cols[kTile + col]),
                   fmaxf(lds_cols[2 * kTile + col], lds_cols[3 * kTile + col]));
  }
}

__device__ __forceinline__ float tile_max(const Tile& t, float* lds4) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, row_partial_max(t, i));
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) lds4[threadIdx.x >> 6] = m;
  __syncthreads();
  return fmaxf(fmaxf(lds4[0], lds4[1]), fmaxf(lds4[2], lds4[3]));
}

// The quotient for units of any scale, out of line: only waves holding a
// unit with S < 2^-90 call it, and keeping its IEEE divisions out of the
// kernel body keeps the common path's register use low.
__device__ __noinline__ float slow_quotient(float x, float s, float r) {
  return quotient(x, UnitScale{s, r, s >= 0x1p-90f});
}

// Which of a thread's 8 x 8 elements share a unit: its rows, its columns, or
// all of them.
enum UnitMap { kUnitRow, kUnitCol, kUnitOne };

// Codes of a thread's 8 x 8 patch (E4M3, or E5M2 when E5), two bytes per
// conversion: byte j of
// packed[i][j / 4] is element (i, j), with the unit scales su (S) and ru
// (1/S) indexed by row, by column, or [0].  The reciprocal-based quotient
// holds for S >= 2^-90 (see quotient()); waves whose units all satisfy it
// take the branch-free path.
template <int MAP, bool E5>
__device__ __forceinline__ void encode_patch(const Tile& t, const float (&su)[8], const float (&ru)[8],
                                             uint32_t (&packed)[8][2]) {
  bool fast = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) fast = fast && su[i] >= 0x1p-90f;
  auto encode_all = [&](auto qf) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float q[4];
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const int j = h * 4 + jj;
          const int u = MAP == kUnitRow ? i : (MAP == kUnitCol ? j : 0);
          q[jj] = qf(t.v[i][j], su[u], ru[u]);
        }
        uint32_t w = fp8_pack2<E5, false>(q[0], q[1], 0u);
        packed[i][h] = fp8_pack2<E5, true>(q[2], q[3], w);
      }
    }
  };
  if (__all(fast))
    encode_all([](float x, float s_, float r_) { return fast_quotient(x, s_, r_); });
  else
    encode_all([](float x, float s_, float r_) { return slow_quotient(x, s_, r_); });
}

// The per-unit constants of a unit whose S is known (the cast pass of the
// multi-tile granularities): the same values unit_scale gives for its amax.
__device__ __forceinline__ UnitScale unit_of_scale(float s) { return UnitScale{s, 1.0f / s, s >= 0x1p-90f}; }

// Per-unit scales when a thread's eight rows are eight units shared by the
// 16 lanes of its DPP row: lane cc of the row group holds the amax of row
// cc % 8, computes that unit's S and 1/S (two IEEE divisions), and the
// group exchanges them by lane shuffles.
template <bool E5, bool KNOWN = false>
__device__ __forceinline__ void share_row_units(float amax, bool pow2, UnitScale& mine, float (&su)[8],
                                                float (&ru)[8]) {
  const int lane = threadIdx.x & 63;
  mine = KNOWN ? unit_of_scale(amax) : unit_scale_fmt<E5>(amax, pow2);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    su[i] = __shfl(mine.s, (lane & 48) | i, 64);
    ru[i] = __shfl(mine.r, (lane & 48) | i, 64);
  }
}

// Per-unit scales when a thread's eight columns are eight units: thread
// (rg < 8, cc) holds the amax of column 8 cc + rg, computes its S and 1/S,
// and the block exchanges them through LDS (the upper half of lds_red, after
// every read of its lower half).
template <bool E5, bool KNOWN = false>
__device__ __forceinline__ void share_col_units(float amax, bool pow2, float* lds_red, UnitScale& mine,
                                                float (&su)[8], float (&ru)[8]) {
  const int cc = threadIdx.x & 15, rg = threadIdx.x >> 4;
  mine = KNOWN ? unit_of_scale(amax) : unit_scale_fmt<E5>(amax, pow2);
  float2* lds_su = reinterpret_cast<float2*>(lds_red + 2 * kTile);
  __syncthreads();
  if (rg < 8) lds_su[cc * 8 + rg] = make_float2(mine.s, mine.r);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 v = lds_su[cc * 8 + j];
    su[j] = v.x;
    ru[j] = v.y;
  }
}

// The 1x128 amax of the row this lane computes (row cc % 8 of its eight):
// each tile row is one 128-column unit spread over a 16-lane DPP row.
__device__ __forceinline__ float block_row_amax(const Tile& t) {
  const int cc = threadIdx.x & 15;
  float am[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) am[i] = row16_max(row_partial_max(t, i));
  float amax = am[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) amax = (cc & 7) == i ? am[i] : amax;
  return amax;
}

// Codes of the thread's 8 x 8 patch in the input's layout: rows row0 ..
// row0+7, columns c .. c+7.
__device__ __forceinline__ void store_patch(const uint32_t (&packed)[8][2], uint8_t* codes, int64_t ldc, int64_t rows,
                                            int64_t cols, int64_t row0, int64_t c) {
  if (c < cols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = row0 + i;
      if (r < rows) *reinterpret_cast<uint2*>(codes + r * ldc + c) = make_uint2(packed[i][0], packed[i][1]);
    }
  }
}

// Codes of a 128 x 128 tile at (r0, c0) written transposed, codes[c][r],
// through LDS: LDS row = tile column (128 bytes = 16 chunks of 8 rows);
// chunk rg of LDS row 8*cc+j is stored at chunk rg ^ cc, which spreads the
// 16 lanes of a DPP row over all 32 banks.  Each output row then goes out as
// 16-byte pieces.
__device__ __forceinline__ void store_patch_transposed(const uint32_t (&packed)[8][2], uint64_t* lds_t,
                                                       uint8_t* codes, int64_t ldc, int64_t rows, int64_t cols,
                                                       int64_t r0, int64_t c0) {
  const int cc = threadIdx.x & 15, rg = threadIdx.x >> 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) lo |= ((packed[i][j >> 2] >> (8 * (j & 3))) & 0xffu) << (8 * i);
#pragma unroll
    for (int i = 4; i < 8; ++i) hi |= ((packed[i][j >> 2] >> (8 * (j & 3))) & 0xffu) << (8 * (i - 4));
    const int lrow = cc * 8 + j;
    lds_t[lrow * 16 + (rg ^ cc)] = (uint64_t)lo | ((uint64_t)hi << 32);
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int orow = p * 32 + (threadIdx.x >> 3);  // tile column = output row
    const int qd = threadIdx.x & 7;                // 16-byte chunk of the output row
    const int sw = orow >> 3;
    const uint64_t a0 = lds_t[orow * 16 + ((2 * qd) ^ sw)];
    const uint64_t a1 = lds_t[orow * 16 + ((2 * qd + 1) ^ sw)];
    const int64_t oc = c0 + orow;
    const int64_t orr = r0 + qd * 16;
    if (oc < cols && orr < rows)
      *reinterpret_cast<uint4*>(codes + oc * ldc + orr) =
          make_uint4((uint32_t)a0, (uint32_t)(a0 >> 32), (uint32_t)a1, (uint32_t)(a1 >> 32));
  }
}

}  // namespace quant_detail

}  // namespace fp8q
