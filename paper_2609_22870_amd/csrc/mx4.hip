// MXFP4 on gfx950: E2M1 codes (1.2.1, bias 1: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with a
// power-of-two scale per unit of 32 elements of a row, in an E8M0 byte.
//
//   S = 2^(floor(log2 amax) - 2), at least 2^-127; 1 for a unit of zeros
//   code = the nearest of E2M1 to x / S, ties to even, magnitudes above 6 to 6
//
// S is the OCP MX rule: amax / S lies in [4, 8), and what exceeds 6 (with a quarter of the
// mantissas) goes to 6.  (The smallest S that clamps nothing has the larger error: root mean
// square 11.53% of normal values and 13.9% of Student-t ones with 4 degrees, here 11.48% and
// 13.2%.)  x / S is exact, so a code is rounded once.  A unit that holds a NaN or an infinity gets the
// byte 255, E8M0's NaN, which a product and the values carry on.
//
// Bound by HBM: 2 bytes read and 17/32 written an element, the other way round for the values
// (12288 x 4096: codes 22.3 us, 5.7 TB/s, values 21.2, 6.0).
#include "device_common.h"
#include "rollout.h"

namespace fp8q {

namespace mx4_detail {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef unsigned short v2us __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));

// A workgroup's tile: 4 R rows, R a wave, by 512 columns.
constexpr int kThreads = 256, kCols = 512;

// The larger halves of both.
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_elementwise_max(__builtin_bit_cast(v2us, a), __builtin_bit_cast(v2us, b)));
}

// The maximum over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true);
  m = m > o ? m : o;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true);
  return m > o ? m : o;
}

// The scale byte of a unit from the bf16 bits of its largest magnitude (exponent fields: S's
// is amax's less 2).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  const int e = (int)(amax >> 7);
  const int b = e - 2 < 0 ? 0 : e - 2;
  return amax == 0 ? 127u : (e == 255 ? 255u : (uint32_t)b);
}

// Eight bf16 values to codes, by the hardware's conversion (two at a time, by the scale's
// exponent field).
__device__ __forceinline__ uint32_t pack8(const uint4& v, float s) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.x), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.y), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.z), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.w), s, 3);
  return c;
}

// 16 bytes at any even address: the hardware takes them in one access (1001 x 5001, quantized
// 7.9 us element by element, here 4.4; values 9.8 and 5.4).
typedef v4u v4u_at2 __attribute__((aligned(2)));

// Elements c .. c + 7 of a row of n, zeros past its end.  WIDE: aligned rows.
template <bool WIDE>
__device__ __forceinline__ uint4 load8(const uint16_t* row, int64_t c, int64_t n) {
  if (c + 8 <= n) {
    const v4u q = WIDE ? __builtin_nontemporal_load(reinterpret_cast<const v4u*>(row + c))
                       : *reinterpret_cast<const v4u_at2*>(row + c);
    return make_uint4(q[0], q[1], q[2], q[3]);
  }
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < n) w[e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Lane l of a wave takes the eight elements from 8 l on, four lanes a unit, in rows w, w + 4, ...
// of the workgroup's; the scale bytes meet in LDS, so that those of its rows leave together.
template <bool WIDE, int R>
__global__ __launch_bounds__(kThreads) void quantize_mx4_kernel(Mx4Args a, int tiles_c) {
  constexpr int kRows = 4 * R;
  __shared__ __attribute__((aligned(16))) uint8_t bytes[2][kRows][8];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const int64_t r0 = tr * kRows, c0 = tc * kCols, c = c0 + lane * 8, padded = mx4_padded(a.cols);
  uint4 v[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t r = r0 + wave + 4 * i;
    v[i] = make_uint4(0, 0, 0, 0);
    if (r < a.rows) v[i] = load8<WIDE>(a.x + r * a.ldx, c, a.cols);
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t r = r0 + wave + 4 * i;
    constexpr uint32_t kAbs = 0x7fff7fffu;
    const uint32_t m = pk_max(pk_max(v[i].x & kAbs, v[i].y & kAbs), pk_max(v[i].z & kAbs, v[i].w & kAbs));
    const uint32_t amax = quad_max((m >> 16) > (m & 0xffffu) ? m >> 16 : m & 0xffffu);
    const uint32_t b = scale_byte(amax);
    const uint32_t code = pack8(v[i], __uint_as_float(b << 23));
    if (r < a.rows && c < padded) *reinterpret_cast<uint32_t*>(a.codes + r * a.ldc + c / 2) = code;
    if ((lane & 3) == 0) bytes[lane >> 5][wave + 4 * i][(lane >> 2) & 7] = (uint8_t)b;
  }
  __syncthreads();
  if (t < 2 * kRows) {
    const int64_t piece = tc * 2 + t / kRows, r = r0 + t % kRows;
    if (r < a.rows && piece * kMxPiece < padded)
      *reinterpret_cast<uint2*>(a.scales + (piece * a.rows + r) * 8) =
          *reinterpret_cast<const uint2*>(bytes[t / kRows][t % kRows]);
  }
}

// The values of codes: a lane eight elements of each of its rows, as above.
template <bool WIDE, int R>
__global__ __launch_bounds__(kThreads) void dequantize_mx4_kernel(Mx4ValuesArgs a, int tiles_c) {
  constexpr int kRows = 4 * R;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const int64_t r0 = tr * kRows, c = tc * kCols + lane * 8;
  if (c >= a.cols) return;
  uint32_t code[R], b[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t r = r0 + wave + 4 * i;
    code[i] = b[i] = 0;
    if (r < a.rows) {
      code[i] = *reinterpret_cast<const uint32_t*>(a.codes + r * a.ldc + c / 2);
      b[i] = a.scales[(c / kMxPiece * a.rows + r) * 8 + c / kMxUnit % 8];
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t r = r0 + wave + 4 * i;
    if (r >= a.rows) break;
    // (the byte 255 is NaN: fp32's field 255 with a mantissa bit; 0 is 2^-127, an fp32 subnormal)
    const float s = __uint_as_float(b[i] == 255 ? 0x7fc00000u : (b[i] == 0 ? 0x00400000u : b[i] << 23));
    uint32_t w[4];
    auto two = [&](auto sel) {
      // E2M1 as fp32: an exponent field of 0 is 0 or 0.5
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t q = code[i] >> (8 * decltype(sel)::value + 4 * e) & 15u, mag = q & 7u;
        const float m = mag < 2 ? 0.5f * (float)mag : __uint_as_float((126u + (mag >> 1)) << 23 | (mag & 1) << 22);
        f[e] = (q & 8u ? -m : m) * s;
      }
      w[decltype(sel)::value] = __builtin_bit_cast(uint32_t, v2bf{(__bf16)f[0], (__bf16)f[1]});
    };
    two(std::integral_constant<int, 0>{});
    two(std::integral_constant<int, 1>{});
    two(std::integral_constant<int, 2>{});
    two(std::integral_constant<int, 3>{});
    uint16_t* const to = a.y + r * a.ldy + c;
    if (c + 8 <= a.cols) {
      const v4u q = {w[0], w[1], w[2], w[3]};
      if (WIDE)
        __builtin_nontemporal_store(q, reinterpret_cast<v4u*>(to));
      else
        *reinterpret_cast<v4u_at2*>(to) = q;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < a.cols) to[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
  }
}

// Eight rows a wave, in flight together; two where that leaves few workgroups, whose loads then wait
// for less (1001 x 5000 7.5 us with eight rows, with two 4.0; its values 7.2 and 4.8).
template <typename F>
hipError_t with_rows(int64_t rows, int64_t cols, F&& launch) {
  const int tiles_c = (int)((cols + kCols - 1) / kCols);
  const int64_t tiles = (rows + 31) / 32 * tiles_c;
  // (a launch has less than 2^32 threads: the ABI refuses more tiles)
  if (tiles <= 1024)
    launch(std::integral_constant<int, 2>{}, (unsigned)((rows + 7) / 8 * tiles_c), tiles_c);
  else
    launch(std::integral_constant<int, 8>{}, (unsigned)tiles, tiles_c);
  return hipGetLastError();
}

}  // namespace mx4_detail

using namespace mx4_detail;

hipError_t launch_quantize_mx4(const Mx4Args& a, hipStream_t s) {
  return with_rows(a.rows, a.cols, [&](auto r, unsigned grid, int tiles_c) {
    constexpr int R = decltype(r)::value;
    if (((uintptr_t)a.x & 15) == 0 && a.ldx % 8 == 0)
      quantize_mx4_kernel<true, R><<<grid, kThreads, 0, s>>>(a, tiles_c);
    else
      quantize_mx4_kernel<false, R><<<grid, kThreads, 0, s>>>(a, tiles_c);
  });
}

hipError_t launch_dequantize_mx4(const Mx4ValuesArgs& a, hipStream_t s) {
  return with_rows(a.rows, a.cols, [&](auto r, unsigned grid, int tiles_c) {
    constexpr int R = decltype(r)::value;
    if (((uintptr_t)a.y & 15) == 0 && a.ldy % 8 == 0)
      dequantize_mx4_kernel<true, R><<<grid, kThreads, 0, s>>>(a, tiles_c);
    else
      dequantize_mx4_kernel<false, R><<<grid, kThreads, 0, s>>>(a, tiles_c);
  });
}

}  // namespace fp8q
