// Device helpers shared by the fp8q kernels (gfx950 / CDNA4, wave64).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace fp8q {

constexpr float kE4M3Max = 448.0f;     // largest finite OCP E4M3 magnitude
constexpr float kE5M2Max = 57344.0f;   // largest finite OCP E5M2 magnitude

// F_max of the code format: E4M3, or E5M2 (E5 = true, the gradient variant).
template <bool E5>
constexpr float fp8_max() { return E5 ? kE5M2Max : kE4M3Max; }

// bf16 halves of a packed dword, widened exactly to fp32.
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Per-unit constants of Eq. 3: the scale S = RN32(amax / F_max) (1 if that
// is 0), its correctly rounded reciprocal, and whether the reciprocal-based
// quotient below is exact for this S.
struct UnitScale {
  float s;
  float r;
  bool fast;
};

__device__ __forceinline__ UnitScale unit_scale(float amax, float fmax = kE4M3Max) {
  UnitScale u;
  float s = amax / fmax;      // IEEE division (correctly rounded)
  u.s = (s == 0.0f) ? 1.0f : s;
  u.r = 1.0f / u.s;           // IEEE division (correctly rounded)
  u.fast = u.s >= 0x1p-90f;
  return u;
}

// The power-of-two variant: S = the smallest power of two with F_max S >=
// amax, at least 2^-127 (the E8M0 range of the matrix instructions' block
// scales), and 1 when amax is 0.  Then |x| / S <= F_max and x / S is exact.
// Both maxima are 7/8 of a power of two, 448 = (7/8) 2^9 and 57344 =
// (7/8) 2^16: with amax = m 2^e (m in [0.5, 1)), amax / F_max =
// (8 m / 7) 2^(e - p), and 8 m / 7 <= 1 exactly when m <= 7/8.
__device__ __forceinline__ UnitScale unit_scale_pow2(float amax, int p = 9) {
  UnitScale u;
  if (amax == 0.0f) {
    u.s = 1.0f;
  } else {
    int e;
    const float m = frexpf(amax, &e);
    int k = e - p + (m > 0.875f ? 1 : 0);
    k = k < -127 ? -127 : k;
    u.s = ldexpf(1.0f, k);
  }
  u.r = 1.0f / u.s;  // exact: a power of two
  u.fast = u.s >= 0x1p-90f;
  return u;
}

__device__ __forceinline__ UnitScale unit_scale(float amax, bool pow2) {
  return pow2 ? unit_scale_pow2(amax) : unit_scale(amax);
}

// The same for the code format E4M3 or E5M2.
template <bool E5>
__device__ __forceinline__ UnitScale unit_scale_fmt(float amax, bool pow2) {
  return pow2 ? unit_scale_pow2(amax, E5 ? 16 : 9) : unit_scale(amax, fp8_max<E5>());
}

// The same scale without IEEE divisions, for kernels whose every lane forms its
// units' own: with r = RN(1 / F_max), q = RN(a r) and the exact residual e = a -
// q F_max, RN(q + e r) is RN32(a / F_max) for every a in the normal range.  The
// hardware's reciprocal of S, good to an ulp, is RN32(1 / S) after one Newton step, but for
// the mantissa of all ones, where the quotient of a power of two alone, no middle
// between codes, is an ulp off: the quotients' codes are those of RN32(x / S).  (Both are
// tested on the CPU for every mantissa.)  Units with a smaller amax (zero among them)
// take the division, and hand the quotient x and S both times 2^64, exactly, so that
// every unit's quotients are the same three instructions.
struct CodeScale {
  float s;     // S
  float d, r;  // lift S and its reciprocal
  float lift;  // 1 or 2^64: x / S = (lift x) / d
};

__device__ __noinline__ inline CodeScale small_code_scale(float amax, float fmax) {
  const float s = amax / fmax;
  if (s == 0.0f) return CodeScale{1.0f, 1.0f, 1.0f, 1.0f};
  const float d = s * 0x1p64f;
  return CodeScale{s, d, 1.0f / d, 0x1p64f};
}

template <bool E5>
__device__ __forceinline__ CodeScale code_scale(float amax, bool pow2) {
  if (pow2) {
    const float s = unit_scale_pow2(amax, E5 ? 16 : 9).s;
    const float lift = s < 0x1p-90f ? 0x1p64f : 1.0f, d = s * lift;
    return CodeScale{s, d, 1.0f / d, lift};
  }
  constexpr float kMax = fp8_max<E5>(), kInv = 1.0f / kMax;
  CodeScale u;
  const float q = amax * kInv;
  u.s = u.d = __builtin_fmaf(__builtin_fmaf(-q, kMax, amax), kInv, q);
  const float r = __builtin_amdgcn_rcpf(u.s);
  u.r = __builtin_fmaf(__builtin_fmaf(-u.s, r, 1.0f), r, r);
  u.lift = 1.0f;
  if (amax < 0x1p-64f) u = small_code_scale(amax, kMax);
  return u;
}

// RN32(x / S) for a bf16 x of the unit whose scale is u.  For S >= 2^-90 the
// quotient is formed from the reciprocal with one residual correction,
//   q0 = RN(x r),  e = RN(q0 S - x) (one FMA),  q = RN(q0 - e r) (one FMA);
// over every pair of a bf16 amax and a bf16 x with |x| <= amax, both signs,
// this gives the same E4M3 code as the correctly rounded quotient (checked
// exhaustively on the CPU, and on the GPU against the oracle).  The residual
// is taken as q0 S - x, not x - q0 S, so that x = -0 keeps its sign: the
// exact zero residual is +0 and -(+0) r + (-0) = -0.  Smaller S take the
// IEEE division.
__device__ __forceinline__ float fast_quotient(float x, float s, float r) {
  const float q0 = x * r;
  const float e = __builtin_fmaf(q0, s, -x);
  return __builtin_fmaf(-e, r, q0);
}

__device__ __forceinline__ float quotient(float x, const UnitScale& u) {
  if (u.fast) return fast_quotient(x, u.s, u.r);
  return x / u.s;
}

// Q_FP8 of two fp32 values into the low (HI=false) or high 16 bits of
// `old`: clamp to +-448, then the hardware E4M3 conversion, which rounds to
// nearest even and keeps the sign of zero.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_pack2(float a, float b, uint32_t old) {
  float ca = __builtin_amdgcn_fmed3f(a, -kE4M3Max, kE4M3Max);
  float cb = __builtin_amdgcn_fmed3f(b, -kE4M3Max, kE4M3Max);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(ca, cb, (int)old, HI);
}

// The E5M2 form: clamp to +-57344, then the hardware E5M2 conversion (round
// to nearest even, sign of zero kept); never an infinity.
template <bool HI>
__device__ __forceinline__ uint32_t e5m2_pack2(float a, float b, uint32_t old) {
  float ca = __builtin_amdgcn_fmed3f(a, -kE5M2Max, kE5M2Max);
  float cb = __builtin_amdgcn_fmed3f(b, -kE5M2Max, kE5M2Max);
  return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(ca, cb, (int)old, HI);
}

// x lifted for its quotient by u, and held to F_max S: where S is an fp32 subnormal of
// few bits it may be up to a third below amax / F_max, and larger quotients clamp.
// (Units that need no lift have a normal S, within 2^-24 of amax / F_max.  A NaN stays.)
template <bool E5>
__device__ __forceinline__ float lifted_value(float x, const CodeScale& u) {
  const float v = x * u.lift, most = fp8_max<E5>() * u.d;
  return fabsf(v) > most ? copysignf(most, v) : v;
}

// The conversion without the clamp, for quotients by a CodeScale: |x / S| is at
// most F_max (1 + 2^-23), which rounds to F_max, by S itself where it is normal and by
// lifted_value where it is not.
template <bool E5, bool HI>
__device__ __forceinline__ uint32_t code_pack2(float a, float b, uint32_t old) {
  return E5 ? (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(a, b, (int)old, HI)
            : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HI);
}

template <bool E5, bool HI>
__device__ __forceinline__ uint32_t fp8_pack2(float a, float b, uint32_t old) {
  return E5 ? e5m2_pack2<HI>(a, b, old) : e4m3_pack2<HI>(a, b, old);
}

// Max over the 16 lanes of a DPP row (lanes 16k .. 16k+15).  Each step
// combines a lane with a partner in the same row; after quad swaps the four
// lanes of a quad agree, the half-row mirror joins the two quads of each half,
// the row mirror joins the two halves.
__device__ __forceinline__ float row16_max(float v) {
  int b = __float_as_int(v);
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(b, b, 0xB1, 0xF, 0xF, false)));  // quad [1,0,3,2]
  b = __float_as_int(v);
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(b, b, 0x4E, 0xF, 0xF, false)));  // quad [2,3,0,1]
  b = __float_as_int(v);
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(b, b, 0x141, 0xF, 0xF, false)));  // row_half_mirror
  b = __float_as_int(v);
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(b, b, 0x140, 0xF, 0xF, false)));  // row_mirror
  return v;
}

// Max over the four DPP rows of the wave for lanes with equal (lane % 16).
__device__ __forceinline__ float across_rows_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  v = fmaxf(v, __shfl_xor(v, 32, 64));
  return v;
}

// A value of the lane 16 (32) lanes away and this lane's, in either order: the
// same pair in both lanes.  One instruction of the vector ALU each, where a shuffle
// goes through LDS.
__device__ __forceinline__ float2 with_lane16(float v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return make_float2(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
// The larger magnitude of the two.
__device__ __forceinline__ float magnitude_max(float2 p) {
  const uint32_t a = __float_as_uint(p.x), b = __float_as_uint(p.y);
  return __uint_as_float(a > b ? a : b);
}
__device__ __forceinline__ float2 with_lane32(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return make_float2(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// The maximum of magnitudes over the 16 lanes of a DPP row, as integers (the same
// order): each step is one instruction, where a float maximum of shuffled bits
// needs the move and a canonicalization of its own.
__device__ __forceinline__ float row16_magnitude_max(float v) {
  uint32_t m = __float_as_uint(v);
  auto step = [&](auto ctrl) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, decltype(ctrl)::value, 0xF, 0xF, true);
    m = m > o ? m : o;
  };
  step(std::integral_constant<int, 0xB1>{});   // quad [1,0,3,2]
  step(std::integral_constant<int, 0x4E>{});   // quad [2,3,0,1]
  step(std::integral_constant<int, 0x141>{});  // row_half_mirror
  step(std::integral_constant<int, 0x140>{});  // row_mirror
  return __uint_as_float(m);
}

__device__ __forceinline__ float wave_max(float v) { return across_rows_max(row16_max(v)); }

// The sum over 4, 8, 16 or 64 neighbouring lanes: every lane gets the same bits
// (each step adds the same pair in both partners).
template <int N = 64>
__device__ __forceinline__ float wave_sum(float v) {
  static_assert(N == 4 || N == 8 || N == 16 || N == 64);
  auto step = [&](auto ctrl) {
    const int b = __float_as_int(v);
    v += __int_as_float(__builtin_amdgcn_update_dpp(b, b, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  step(std::integral_constant<int, 0xB1>{});                          // quad [1,0,3,2]
  step(std::integral_constant<int, 0x4E>{});                          // quad [2,3,0,1]
  if constexpr (N >= 8) step(std::integral_constant<int, 0x141>{});   // row_half_mirror
  if constexpr (N >= 16) step(std::integral_constant<int, 0x140>{});  // row_mirror
  if constexpr (N == 64) {
    float2 p = with_lane16(v);
    p = with_lane32(p.x + p.y);
    v = p.x + p.y;
  }
  return v;
}

}  // namespace fp8q
