// Log-probabilities of the taken tokens, and the clipped policy loss with a KL
// term, forward and backward, from the logits of each token on gfx950.
//
// With z = x / temperature over a row of V logits, and the taken token a,
//   lse = log sum exp(z),  p = exp(z - lse),  logp = z_a - lse,
//   entropy = lse - sum p z,
//   r = exp(logp - logp_old),  d = logp_ref - logp,
//   l = -w min(r A, clip(r, low, high) A) + beta (exp(d) - d - 1),
//   l' = dl / dlogp = -w A r [r A <= clip(r) A] + beta (1 - exp(d)),
//   loss = sum c l,  dx_j = c l' / temperature (delta_aj - p_j)
// over the tokens with weight c != 0 and a inside the vocabulary; all other
// rows are not read: their results and gradients are zero.
//
// Bound by HBM: the logits read once, the gradient written once.  So a
// workgroup holds a whole row in registers between the two (131072 bf16 logits
// are half of a CU's registers), takes the running maximum, sum and entropy sum
// while its pieces arrive, and writes the gradient from the registers.  Longer
// rows read what exceeds them again.  Too few rows to fill the chip are split
// over several workgroups, which leave their sums in a workspace, and a second
// kernel joins them.  Everything is in base 2 (one fused multiply-add and one
// v_exp_f32 an element), with the temperature in the factor log2(e) / t.  4096 x
// 65536 bf16 with the gradient 199 us (5.4 TB/s); 64 x 131072 without 11.4 us, its two
// kernels 8 and 2 of them.
#include <type_traits>

#include "device_common.h"
#include "ops.h"

namespace fp8q {

namespace loss_detail {

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

// What the loss needs of a token besides its logits, and what its row gets.
struct Token {
  float k;  // c l' / temperature
  float logp, entropy, term;
};

__device__ __forceinline__ Token token_of(const LossArgs& a, int64_t row, const Sums& sums, float x, bool grad) {
  Token o{};
  const float log_s = logf(sums.s);
  // u ln 2 - log s; entropy = log s - ln 2 q / s, both relative to the maximum's exponent
  const float c = a.inv_temperature * kLog2e;
  const Exponent exponent(c, sums.m);
  const float u = exponent.c == c ? exponent(x) : (x - sums.m) * c;
  o.logp = __builtin_fmaf(u, kLn2, -log_s);
  o.entropy = log_s - kLn2 * (sums.q / sums.s);
  if (!grad) return o;
  const float low = a.clip ? (float)a.clip->l_new : a.clip_low, high = a.clip ? (float)a.clip->h_new : a.clip_high;
  const float adv = a.adv[row], w = a.w_tis ? a.w_tis[row] : 1.0f, weight = a.weight[row];
  // (the ratio stays finite, and w A is formed first: an advantage or weight of zero
  // then takes nothing from a ratio that fp32 does not hold)
  const float e = expf(o.logp - a.logp_old[row]), r = e > 0x1.fffffep127f ? 0x1.fffffep127f : e;
  const float bounded = fminf(fmaxf(r, low), high), wa = w * adv;
  const bool clipped = r * adv > bounded * adv;
  float l = -wa * (clipped ? bounded : r);
  float slope = clipped ? 0.0f : -wa * r;
  if (a.logp_ref) {
    const float d = a.logp_ref[row] - o.logp, m = expm1f(d);
    l += a.beta * (m - d);
    slope -= a.beta * m;
  }
  o.term = weight * l;
  o.k = weight * slope * a.inv_temperature;
  return o;
}

// Whether the row counts: its token lies in the vocabulary and, for the loss,
// its weight is not zero.
__device__ __forceinline__ bool counts(const LossArgs& a, int64_t row, int64_t token, bool grad) {
  return token >= 0 && token < a.V && (!grad || a.weight[row] != 0.0f);
}

// A row's gradient: dx_j = (delta - p) k, p = 2^u / s, ks = k / s.
template <bool F32>
struct Gradient {
  using P = Piece<F32>;
  uint8_t* out;
  bool aligned;  // as the row of logits is, so that pieces go out whole
  int head, token;
  Exponent u;
  float k, ks;
  __device__ __forceinline__ Gradient(const LossArgs& a, int64_t row, const Row<F32>& x, int64_t tok, const Sums& sums,
                                      float kk)
      : u(a.inv_temperature * kLog2e, sums.m) {
    out = static_cast<uint8_t*>(a.dlogits) + row * a.ldd * P::kSize;
    aligned = (((uintptr_t)out ^ (uintptr_t)x.base) & 15) == 0;
    head = x.head;
    token = (int)tok;
    k = kk;
    ks = kk / sums.s;
  }
  __device__ __forceinline__ float of(float x, bool taken) const {
    return (taken ? k : 0.0f) - ks * __builtin_amdgcn_exp2f(u(x));
  }
  // of piece j0 + t, where that is below last
  __device__ __forceinline__ void put(const uint4& p, int j0, int last, unsigned t) const {
    if ((int)t >= last - j0) return;
    float v[P::kN];
    P::widen(p, v);
#pragma unroll
    for (int e = 0; e < P::kN; ++e) v[e] = -ks * __builtin_amdgcn_exp2f(u(v[e]));
    const unsigned at = (unsigned)(token - head - j0 * P::kN) - t * P::kN;
    if (at < (unsigned)P::kN) {
#pragma unroll
      for (int e = 0; e < P::kN; ++e) v[e] += at == (unsigned)e ? k : 0.0f;
    }
    const uint4 g = P::narrow(v);
    uint8_t* const to = out + head * P::kSize + (int64_t)j0 * 16;
    if (aligned) {
      // past the caches, which keep what is still to be read (4096 x 32000 bf16 108 -> 86
      // us, 4096 x 65536 fp32 490 -> 425, 8192 x 131072 bf16 853 -> 845; with the dual
      // quantizer that reads the gradient next, 128 x 32768 bf16 22.2 -> 20.5, 1024 rows 54.4 ->
      // 54.7, 4096 x 65536 448 -> 445)
      __builtin_nontemporal_store(v4u{g.x, g.y, g.z, g.w}, reinterpret_cast<v4u*>(to + t * 16u));
    } else {
      const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
      for (int e = 0; e < P::kN; ++e) {
        if constexpr (F32)
          reinterpret_cast<uint32_t*>(to)[t * 4u + e] = w[e];
        else
          reinterpret_cast<uint16_t*>(to)[t * 8u + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
};

// A row's gradient of zeros, by THREADS threads.
template <bool F32, int THREADS>
__device__ __forceinline__ void store_zeros(const LossArgs& a, int64_t row, int64_t first, int64_t last, int t) {
  using P = Piece<F32>;
  uint8_t* const out = static_cast<uint8_t*>(a.dlogits) + row * a.ldd * P::kSize;
  for (int64_t i = first + t; i < last; i += THREADS) P::store(out, i, 0.0f);
}

// One workgroup a row.  GRAD: the first NV pieces of every thread stay in
// registers for the gradient; the others are read again.
template <bool F32, int THREADS, int NV, bool GRAD>
__global__ __launch_bounds__(THREADS) void row_kernel(LossArgs a) {
  using P = Piece<F32>;
  constexpr int W = THREADS / 64, kChunk = NV % 4 == 0 ? 4 : 3;
  __shared__ Sums parts[W];
  __shared__ Token shared;
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int64_t token = a.tokens[row];
  if (!counts(a, row, token, GRAD)) {  // the whole workgroup
    if (GRAD) store_zeros<F32, THREADS>(a, row, 0, a.V, t);
    if (t == 0) {
      a.logp[row] = 0.0f;
      a.entropy[row] = 0.0f;
      if (GRAD) a.terms[row] = 0.0f;
    }
    return;
  }
  const float c = a.inv_temperature * kLog2e;
  const Row<F32> x(a.logits, a.ld, row, a.V);
  const float mine = P::load(x.base, token);
  const int edge = x.edge(t);
  float ev = kNegInf;
  if (edge >= 0) ev = P::load(x.base, edge);

  uint4 held[NV];
  Sums sums{kNegInf, 0.0f, 0.0f};
  auto fetch = [&](int j0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) held[i] = x.piece(j0 + i * THREADS, x.full, t);
  };
  auto add = [&]() {
#pragma unroll
    for (int i = 0; i < NV; i += kChunk) {
      add_pieces<F32, kChunk>(held + i, c, sums);
      __builtin_amdgcn_sched_barrier(0);  // one chunk's fp32 values live at a time
    }
  };
  // the pieces past the first NV of each thread, if any, then those
  constexpr int kStep = NV * THREADS;
  for (int j0 = kStep; j0 < x.full; j0 += kStep) {
    fetch(j0);
    add();
  }
  fetch(0);
  add();
  if (edge >= 0) sums = join(sums, single(ev, c), c);
  sums = wave_join(sums, c);
  if ((t & 63) == 0) parts[t >> 6] = sums;
  __syncthreads();
  sums = wave_join<W>(parts[t & (W - 1)], c);
  if (t == 0) {
    const Token o = token_of(a, row, sums, mine, GRAD);
    a.logp[row] = o.logp;
    a.entropy[row] = o.entropy;
    if (GRAD) {
      a.terms[row] = o.term;
      shared = o;
    }
  }
  if constexpr (GRAD) {
    __syncthreads();
    const Gradient<F32> g(a, row, x, token, sums, shared.k);
    auto put = [&](int j0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        forget(held[i]);
        g.put(held[i], j0 + i * THREADS, x.full, t);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    put(0);
    for (int j0 = kStep; j0 < x.full; j0 += kStep) {
      fetch(j0);
      put(j0);
    }
    if (edge >= 0) P::store(g.out, edge, g.of(ev, edge == g.token));
  }
}

// Few rows: workgroup (part, row) takes every piece j with j / per == part, and
// part 0 the row's edges.
constexpr int kSplitThreads = 256;

template <bool F32, bool GRAD>
__global__ __launch_bounds__(kSplitThreads) void split_sums_kernel(LossArgs a, int per) {
  using P = Piece<F32>;
  constexpr int W = kSplitThreads / 64, NV = 8;
  __shared__ Sums shared[W];
  const int t = threadIdx.x;
  const int64_t part = blockIdx.x, row = blockIdx.y;
  if (!counts(a, row, a.tokens[row], GRAD)) return;
  const float c = a.inv_temperature * kLog2e;
  const Row<F32> x(a.logits, a.ld, row, a.V);
  const int first = (int)part * per, last = first + per < x.full ? first + per : x.full;
  Sums sums{kNegInf, 0.0f, 0.0f};
  for (int j0 = first; j0 < last; j0 += NV * kSplitThreads) {
    uint4 held[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) held[i] = x.piece(j0 + i * kSplitThreads, last, t);
    add_pieces<F32, NV>(held, c, sums);
  }
  const int edge = part == 0 ? x.edge(t) : -1;
  if (edge >= 0) sums = join(sums, single(P::load(x.base, edge), c), c);
  sums = wave_join(sums, c);
  if ((t & 63) == 0) shared[t >> 6] = sums;
  __syncthreads();
  sums = wave_join<W>(shared[t & (W - 1)], c);
  if (t == 0) {
    float* const p = a.partials + (row * kLossParts + part) * 4;
    p[0] = sums.m;
    p[1] = sums.s;
    p[2] = sums.q;
    if (part == 0) p[3] = P::load(x.base, a.tokens[row]);  // (dlogits may be written over the logits)
  }
}

// A row's sums from its parts, joined in one order by every wave that asks.
__device__ __forceinline__ Sums joined(const LossArgs& a, int64_t row, int parts) {
  const int lane = threadIdx.x & 63;
  Sums s{kNegInf, 0.0f, 0.0f};
  if (lane < parts) {
    const float* const p = a.partials + (row * kLossParts + lane) * 4;
    s = Sums{p[0], p[1], p[2]};
  }
  return wave_join(s, a.inv_temperature * kLog2e);
}

// The log-probabilities of split rows: a wave a row.
__global__ __launch_bounds__(64) void split_logprobs_kernel(LossArgs a, int parts) {
  const int64_t row = blockIdx.x;
  Token o{};
  if (counts(a, row, a.tokens[row], false))
    o = token_of(a, row, joined(a, row, parts), a.partials[row * kLossParts * 4 + 3], false);
  if (threadIdx.x == 0) {
    a.logp[row] = o.logp;
    a.entropy[row] = o.entropy;
  }
}

// The loss of split rows, by one workgroup: sixteen lanes a row join its parts and
// form its token's term; the terms are added in float64, in a fixed order.
__device__ __forceinline__ void split_loss(const LossArgs& a, int parts) {
  __shared__ double terms[kLossSplitRows];
  const int t = threadIdx.x, lane = t & 15;
  const float c = a.inv_temperature * kLog2e;
  if (t < kLossSplitRows) terms[t] = 0.0;
  __syncthreads();
  for (int r0 = 0; r0 < a.T; r0 += kSplitThreads / 16) {
    const int64_t row = r0 + (t >> 4);
    const bool live = row < a.T && counts(a, row, a.tokens[row], true);
    const float4* const p = reinterpret_cast<const float4*>(a.partials) + row * kLossParts;
    Sums s{kNegInf, 0.0f, 0.0f};
    float x = 0.0f;
    if (live) {
      float4 v[kLossParts / 16];
#pragma unroll
      for (int i = 0; i < kLossParts / 16; ++i)
        v[i] = lane + 16 * i < parts ? p[lane + 16 * i] : make_float4(kNegInf, 0.0f, 0.0f, 0.0f);
      x = a.partials[row * kLossParts * 4 + 3];
#pragma unroll
      for (int i = 0; i < kLossParts / 16; ++i) s = join(s, Sums{v[i].x, v[i].y, v[i].z}, c);
    }
    const float m = row16_max(s.m);
    s = moved(s, m, c);
    s = Sums{m, wave_sum<16>(s.s), wave_sum<16>(s.q)};
    if (live && lane == 0) terms[row] = (double)token_of(a, row, s, x, true).term;
  }
  __syncthreads();
  for (int n = kLossSplitRows / 2; n > 0; n /= 2) {
    if (t < n) terms[t] += terms[t + n];
    __syncthreads();
  }
  if (t == 0) *a.loss = (float)terms[0];
}

// Workgroup (part, row + 1): the gradient of that part; (0, 0): the loss.
template <bool F32>
__global__ __launch_bounds__(kSplitThreads) void split_gradient_kernel(LossArgs a, int per, int parts) {
  using P = Piece<F32>;
  constexpr int NV = 4;
  if (blockIdx.y == 0) {
    if (blockIdx.x == 0) split_loss(a, parts);
    return;
  }
  const int t = threadIdx.x;
  const int64_t part = blockIdx.x, row = (int64_t)blockIdx.y - 1;
  const int64_t token = a.tokens[row];
  const Row<F32> x(a.logits, a.ld, row, a.V);
  const int first = (int)part * per, last = first + per < x.full ? first + per : x.full;
  const int edge = part == 0 ? x.edge(t) : -1;
  if (!counts(a, row, token, true)) {
    store_zeros<F32, kSplitThreads>(a, row, x.head + first * P::kN, x.head + last * P::kN, t);
    if (edge >= 0) P::store(static_cast<uint8_t*>(a.dlogits) + row * a.ldd * P::kSize, edge, 0.0f);
    if (part == 0 && t == 0) a.logp[row] = a.entropy[row] = 0.0f;
    return;
  }
  const Sums sums = joined(a, row, parts);
  const Token o = token_of(a, row, sums, a.partials[row * kLossParts * 4 + 3], true);
  if (part == 0 && t == 0) {
    a.logp[row] = o.logp;
    a.entropy[row] = o.entropy;
  }
  const Gradient<F32> g(a, row, x, token, sums, o.k);
  for (int j0 = first; j0 < last; j0 += NV * kSplitThreads) {
    uint4 held[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) held[i] = x.piece(j0 + i * kSplitThreads, last, t);
#pragma unroll
    for (int i = 0; i < NV; ++i) g.put(held[i], j0 + i * kSplitThreads, last, t);
  }
  if (edge >= 0) P::store(g.out, edge, g.of(P::load(x.base, edge), edge == g.token));
}

// The loss from the tokens' parts, in float64, in a fixed order.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void loss_sum_kernel(const float* terms, int64_t T, float* loss) {
  __shared__ double lds[kSumThreads];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < T; i += kSumThreads) s += (double)terms[i];
  lds[threadIdx.x] = s;
  __syncthreads();
  for (int n = kSumThreads / 2; n > 0; n /= 2) {
    if ((int)threadIdx.x < n) lds[threadIdx.x] += lds[threadIdx.x + n];
    __syncthreads();
  }
  if (threadIdx.x == 0) *loss = (float)lds[0];
}

// Pieces of each of the workgroups that share a row, and their number.
inline int split_parts(int64_t T, int64_t pieces, int& per) {
  int64_t parts = (1024 + T - 1) / T;
  const int64_t most = (pieces + kSplitThreads * 4 - 1) / (kSplitThreads * 4);  // of four pieces a thread or more
  if (parts > most) parts = most;
  if (parts > kLossParts) parts = kLossParts;
  if (parts < 1) parts = 1;
  per = (int)((pieces + parts - 1) / parts);
  return (int)parts;
}

// Whether rows are split over workgroups.  A row in one workgroup takes its CU's
// time: GPU us of a call 6 + 1.05e-4 V (bf16) or 1.7e-4 V (fp32) with the gradient
// and 3 + 6.2e-5 V without; split rows 9 (6) for a launch more, and then the whole
// chip's time, 1.1e-6 (1.7e-6 fp32, 5.4e-7 without the gradient) T V.  Measured, one
// workgroup and split: 33 x 131072 bf16 20.7 and 13.3, 127 rows 24.8 and 33.2; 33 x
// 32000 11.4 and 11.2; 33 x 131072 fp32 34.4 and 15.3, 64 x 32000 13.4 and 14.0;
// log-probabilities of 64 x 131072 12.0 and 9.8, of 127 12.5 and 12.6.
inline bool split_rows(int64_t T, int64_t V, bool f32, bool grad) {
  if (T >= kLossSplitRows) return false;
  const double t = (double)T, v = (double)V;
  if (!grad) return v * (6.2e-5 - 5.4e-7 * t) > 3.0;
  return v * (f32 ? 1.7e-4 - 1.7e-6 * t : 1.05e-4 - 1.1e-6 * t) > 3.0;
}

template <bool F32, bool GRAD>
hipError_t launch_rows(const LossArgs& a, hipStream_t s) {
  constexpr int N = Piece<F32>::kN;
  const int64_t pieces = a.V / N;  // (the most a row has)
  if (split_rows(a.T, a.V, F32, GRAD)) {
    int per;
    const int parts = split_parts(a.T, pieces, per);
    const dim3 grid((unsigned)parts, (unsigned)a.T);
    split_sums_kernel<F32, GRAD><<<grid, kSplitThreads, 0, s>>>(a, per);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if constexpr (GRAD)
      split_gradient_kernel<F32><<<dim3(grid.x, grid.y + 1), kSplitThreads, 0, s>>>(a, per, parts);
    else
      split_logprobs_kernel<<<dim3((unsigned)a.T), 64, 0, s>>>(a, parts);
    return hipGetLastError();
  }
  // The smallest workgroup whose registers hold the row, so that a CU has more rows
  // in flight (bf16: 4096 x 65536 in 512 threads 211 us, in 1024 279; 32768 in 256
  // 113, in 512 132, all with cached stores; log-probabilities of 4096 x 8192 in 256 threads 16, in 512 34).
  const dim3 grid((unsigned)a.T);
  if constexpr (!GRAD) {
    if (pieces <= 4 * 256)
      row_kernel<F32, 256, 4, false><<<grid, 256, 0, s>>>(a);
    else if (pieces <= 8 * 512)
      row_kernel<F32, 512, 8, false><<<grid, 512, 0, s>>>(a);
    else
      row_kernel<F32, 1024, 8, false><<<grid, 1024, 0, s>>>(a);
  } else if (pieces <= 4 * 256) {
    row_kernel<F32, 256, 4, true><<<grid, 256, 0, s>>>(a);
  } else if (pieces <= 8 * 256) {
    row_kernel<F32, 256, 8, true><<<grid, 256, 0, s>>>(a);
  } else if (pieces <= 16 * 256) {
    row_kernel<F32, 256, 16, true><<<grid, 256, 0, s>>>(a);
  } else if (pieces <= 16 * 512) {
    row_kernel<F32, 512, 16, true><<<grid, 512, 0, s>>>(a);
  } else if (pieces <= 16 * 1024) {
    row_kernel<F32, 1024, 16, true><<<grid, 1024, 0, s>>>(a);
  } else {
    row_kernel<F32, 1024, F32 ? 18 : 20, true><<<grid, 1024, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace loss_detail

using namespace loss_detail;

hipError_t launch_logprobs(const LossArgs& a, hipStream_t s) {
  return a.f32 ? launch_rows<true, false>(a, s) : launch_rows<false, false>(a, s);
}

hipError_t launch_policy_loss(const LossArgs& a, hipStream_t s) {
  const hipError_t e = a.f32 ? launch_rows<true, true>(a, s) : launch_rows<false, true>(a, s);
  if (e != hipSuccess || split_rows(a.T, a.V, a.f32, true)) return e;  // (split rows: the loss is there)
  loss_sum_kernel<<<1, kSumThreads, 0, s>>>(a.terms, a.T, a.loss);
  return hipGetLastError();
}

}  // namespace fp8q
