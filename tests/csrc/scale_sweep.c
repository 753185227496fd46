/*
 * Test helper: the arithmetic by which the kernels that form their own units' scales
 * and quotients (device_common.h: code_scale, fast_quotient) do without IEEE
 * divisions, against those divisions.
 *
 *   S = RN(q + e k),  k = RN(1 / F),  q = RN(a k),  e = RN(a - q F)
 *   r = RN(r0 + r0 RN(1 - S r0)),  r0 the hardware's reciprocal: 1 / S to an ulp
 *   x / S = RN(q0 - r RN(q0 S - x)),  q0 = RN(x r)
 *
 * Host fmaf and float products are the same IEEE operations as the kernels'.
 */
#include <math.h>
#include <stdint.h>
#include <string.h>

static float f32(uint32_t b) { float x; memcpy(&x, &b, 4); return x; }
static uint32_t bits(float x) { uint32_t b; memcpy(&b, &x, 4); return b; }

/* Amaxes of every mantissa and the exponent field `exponent` whose scale is not
 * RN(a / fmax). */
uint64_t scale_sweep(float fmax, uint32_t exponent) {
  const float k = 1.0f / fmax;
  uint64_t bad = 0;
  for (uint32_t m = 0; m < 1u << 23; ++m) {
    const float a = f32(exponent << 23 | m);
    const float q = a * k, s = fmaf(fmaf(-q, fmax, a), k, q);
    bad += bits(s) != bits(a / fmax);
  }
  return bad;
}

static float refined(float s, float r0) { return fmaf(fmaf(-s, r0, 1.0f), r0, r0); }

/* Scales 1 <= S < 2 whose refined reciprocal is not RN(1 / S), from either of the
 * two values within an ulp of 1 / S; *last: the last such scale's mantissa. */
uint64_t reciprocal_sweep(uint32_t* last) {
  uint64_t bad = 0;
  for (uint32_t m = 0; m < 1u << 23; ++m) {
    const float s = f32(127u << 23 | m), r = 1.0f / s;
    const float rest = fmaf(-s, r, 1.0f); /* its sign says on which side of r 1 / S lies */
    const float other = f32(bits(r) + (rest > 0.0f) - (rest < 0.0f));
    if (bits(refined(s, r)) != bits(r) || bits(refined(s, other)) != bits(r)) {
      ++bad;
      *last = m;
    }
  }
  return bad;
}

/* The quotients by the scale 2 - 2^-23, whose refined reciprocal is not RN(1 / S):
 * every mantissa of x.  *worst: mantissa of the last x / S that is wrong. */
uint64_t last_scale_sweep(uint32_t* worst) {
  const float s = f32(127u << 23 | 0x7fffff), r = refined(s, 1.0f / s);
  uint64_t bad = 0;
  for (uint32_t m = 0; m < 1u << 23; ++m) {
    const float x = f32(127u << 23 | m), q0 = x * r, q = fmaf(-fmaf(q0, s, -x), r, q0);
    if (bits(q) != bits(x / s)) {
      ++bad;
      *worst = m;
    }
  }
  return bad;
}

/* n pairs of mantissas, x and S in [1, 2), S not the last: quotients that are not
 * RN(x / S). */
uint64_t quotient_sweep(uint64_t n, uint64_t seed) {
  uint64_t bad = 0, z = seed;
  for (uint64_t i = 0; i < n; ++i) {
    z = z * 6364136223846793005ull + 1442695040888963407ull;
    uint32_t ms = (uint32_t)(z >> 41);
    const uint32_t mx = (uint32_t)(z >> 18) & 0x7fffff;
    if (ms == 0x7fffff) ms = 0;
    const float s = f32(127u << 23 | ms), x = f32(127u << 23 | mx), r = 1.0f / s;
    const float q0 = x * r, q = fmaf(-fmaf(q0, s, -x), r, q0);
    bad += bits(q) != bits(x / s);
  }
  return bad;
}
