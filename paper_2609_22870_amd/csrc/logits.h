// Rows of logits in 16-byte pieces, and the running sums of their softmax, for the
// kernels that read them (loss.hip, top.hip).
#pragma once

#include <type_traits>

#include "device_common.h"
#include "ops.h"

namespace fp8q {

namespace logits_detail {

typedef float v2f __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 0x1.715476p+0f, kLn2 = 0x1.62e430p-1f;
constexpr float kNegInf = -__builtin_inff();

// A 16-byte piece of logits as fp32 and back.
template <bool F32>
struct Piece {
  static constexpr int kN = F32 ? 4 : 8;
  static constexpr int kSize = F32 ? 4 : 2;
  static __device__ __forceinline__ void widen(const uint4& p, float (&v)[kN]) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (F32) {
        v[e] = __uint_as_float(w[e]);
      } else {
        v[2 * e] = bf16_lo(w[e]);
        v[2 * e + 1] = bf16_hi(w[e]);
      }
    }
  }
  static __device__ __forceinline__ uint4 narrow(const float (&v)[kN]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (F32)
        w[e] = __float_as_uint(v[e]);
      else
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{v[2 * e], v[2 * e + 1]}), v2bf));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ uint4 nothing() {  // -inf throughout
    const uint32_t w = F32 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
  }
  static __device__ __forceinline__ float load(const uint8_t* row, int64_t i) {
    if constexpr (F32) return reinterpret_cast<const float*>(row)[i];
    return bf16_lo(reinterpret_cast<const uint16_t*>(row)[i]);
  }
  static __device__ __forceinline__ void store(uint8_t* row, int64_t i, float v) {
    if constexpr (F32) {
      reinterpret_cast<float*>(row)[i] = v;
    } else {
      reinterpret_cast<__bf16*>(row)[i] = (__bf16)v;
    }
  }
};

// From here on p is another value to the compiler: it would else keep the fp32
// form of every held piece from the sums to the gradient, and spill.
__device__ __forceinline__ void forget(uint4& p) { asm volatile("" : "+v"(p.x), "+v"(p.y), "+v"(p.z), "+v"(p.w)); }

// The exponents of a row relative to that of its maximum m: u = x c - ref, one fused
// multiply-add, with c = log2(e) / temperature and ref = RN(m c).  What ref is off by
// is the same for every element, so it cancels; but from |m c| = 2^31 on it would
// leave exp2's range (and m c that of fp32, in a row of nothing but the type's lowest
// value, say).  There any other value is 2^7 or more below m's exponent, a weight of
// nothing, so the scale is taken as the power of two that puts m c at 2^40: ref is
// exact, m's own u 0 and every other's weight 0.  Relative to 0 where nothing is
// finite.
struct Exponent {
  float c, ref;
  __device__ __forceinline__ Exponent(float c_, float m) : c(c_) {
    const float base = m == kNegInf ? 0.0f : m;
    ref = base * c;
    const bool wide = !in_range(ref);
    if (__any(wide)) {
      c = wide ? ldexpf(1.0f, min(41 - __builtin_amdgcn_frexp_expf(base), 126)) : c;
      ref = base * c;
    }
  }
  static __device__ __forceinline__ bool in_range(float ref) { return fabsf(ref) < 0x1p31f; }
  __device__ __forceinline__ float operator()(float x) const { return __builtin_fmaf(x, c, -ref); }
};

// The exponent of x relative to m alone, at any range (x <= m, m above -inf).
__device__ __forceinline__ float exponent_below(float x, float m, float c) {
  const float ref = m * c;
  return Exponent::in_range(ref) ? x * c - ref : (x - m) * c;
}

// Running sums of a softmax, over exponents relative to that of the maximum m: s =
// sum 2^u, q = sum 2^u u; m = -inf: nothing finite yet.
struct Sums {
  float m, s, q;
};

// Sums taken to the larger maximum m.
__device__ __forceinline__ Sums moved(const Sums& a, float m, float c) {
  // (one without a finite logit has nothing to move; one with +inf or NaN carries
  // NaN in s)
  const float d = a.m == kNegInf || a.m == m ? 0.0f : fmaxf(exponent_below(a.m, m, c), -1e30f);
  const float f = __builtin_amdgcn_exp2f(d);
  return Sums{m, a.s * f, f * __builtin_fmaf(a.s, d, a.q)};
}

// The sums of both, in either order.
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const Sums x = moved(a, m, c), y = moved(b, m, c);
  return Sums{m, x.s + y.s, x.q + y.q};
}

// The sums of one element (NaN for +inf or NaN).
__device__ __forceinline__ Sums single(float x, float c) {
  const float u = Exponent(c, x)(x), y = __builtin_amdgcn_exp2f(u);
  return Sums{x, y, y * fmaxf(u, -1e30f)};
}

// The sums of N neighbouring lanes (every lane gets the same bits), or of as many
// that every N lanes hold again: all are taken to the common maximum, then added.
template <int N = 64>
__device__ __forceinline__ Sums wave_join(const Sums& a, float c) {
  const float m = wave_max(a.m);
  const Sums x = moved(a, m, c);
  return Sums{m, wave_sum<N>(x.s), wave_sum<N>(x.q)};
}

// Adds K pieces to a thread's sums.
template <bool F32, int K>
__device__ __forceinline__ void add_pieces(uint4* p, float c, Sums& a) {
  using P = Piece<F32>;
  float top = kNegInf;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float v[P::kN];
    P::widen(p[k], v);
#pragma unroll
    for (int e = 0; e < P::kN; ++e) top = fmaxf(top, v[e]);
  }
  const float m = fmaxf(a.m, top);
  a = moved(a, m, c);
  const Exponent exponent(c, m);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    forget(p[k]);
    float v[P::kN];
    P::widen(p[k], v);
#pragma unroll
    for (int e = 0; e < P::kN; ++e) {
      const float u = exponent(v[e]);
      const float x = __builtin_amdgcn_exp2f(u);
      a.s += x;
      a.q = __builtin_fmaf(x, fmaxf(u, -1e30f), a.q);  // (a logit of -inf adds 0, not 0 * -inf)
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A row of logits: `full` aligned 16-byte pieces from element `head` on, and
// before and after them fewer than a piece's elements each, one a thread.
// Everything but the thread's own part of an address is the same in the whole
// workgroup, so a piece's address is a scalar and one 32-bit offset for all
// pieces (64-bit ones for each took the registers that hold the row).
template <bool F32>
struct Row {
  using P = Piece<F32>;
  const uint8_t* base;
  int V, head, full;
  __device__ __forceinline__ Row(const void* logits, int64_t ld, int64_t row, int64_t v) {
    V = (int)v;
    base = static_cast<const uint8_t*>(logits) + row * ld * P::kSize;
    const int lead = (16 - (int)((uintptr_t)base & 15)) % 16 / P::kSize;
    head = lead < V ? lead : V;
    full = (V - head) / P::kN;
  }
  // piece j0 + t, where that is below last
  __device__ __forceinline__ uint4 piece(int j0, int last, unsigned t) const {
    uint4 p = P::nothing();
    if ((int)t < last - j0)
      p = *reinterpret_cast<const uint4*>(base + head * P::kSize + (int64_t)j0 * 16 + t * 16u);
    return p;
  }
  // this thread's single element: its index, or -1
  __device__ __forceinline__ int edge(int t) const { return row_edge(t, V, head, full, P::kN); }
};

}  // namespace logits_detail

}  // namespace fp8q
