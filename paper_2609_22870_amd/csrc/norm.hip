// Root-mean-square norm with the residual's addition, and FP8 output (Eq. 3's
// scales and codes), on gfx950; and its backward pass.
//
//   h = bf16(x + residual)            the residual stream, as it is kept
//   rstd = 1 / sqrt(mean(h^2) + eps)  over the row, in fp32
//   y = h rstd w                      in fp32, rounded once: to bf16, or to
//                                     E4M3 codes of y / S, S = RN32(amax / 448)
//
// The norm is that of the rounded h, so that the backward pass, which has only
// h and rstd, differentiates what the forward pass computed.
//
// Bound by HBM: 7 bytes an element with a residual and codes (x, residual and h
// in bf16, one code), 3 without a residual (16384 x 5120 with both 108 us, 5.5 TB/s).  So a row is read once and held in
// registers between the sum of squares and the output: VPT pieces of 16 bytes
// a thread, THREADS threads a row.  The 16 lanes of a DPP row hold 128
// consecutive elements, one 1x128 unit.
#include <type_traits>

#include "device_common.h"
#include "ops.h"

namespace fp8q {

namespace norm_detail {

typedef float v2f __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t bf16x2_rne(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{lo, hi}), v2bf));
}

__device__ __forceinline__ void widen(const uint4& p, float (&v)[8]) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = bf16_lo(w[e]);
    v[2 * e + 1] = bf16_hi(w[e]);
  }
}

__device__ __forceinline__ uint4 narrow(const float (&v)[8]) {
  return make_uint4(bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7]));
}

// 16 bytes of the streams in and out of a layer: past the caches, which keep the codes
// for the GEMM that follows.  A quantizer that reads dx right after takes it from
// memory then, and the two together are faster all the same but around 64 MB (backward
// pass and dual quantizer, stores past the caches and not: 8 MB of dx 23.6 and 26.2 us, 64
// MB 82.0 and 79.9, 512 MB 590 and 624).
__device__ __forceinline__ uint4 read_once(const uint16_t* p) {
  const v4u v = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void write_once(uint16_t* p, const uint4& v) {
  __builtin_nontemporal_store(v4u{v.x, v.y, v.z, v.w}, reinterpret_cast<v4u*>(p));
}

// From here on p is another value to the compiler: it would else keep the fp32
// form of a held piece across the row's reduction, in twice the registers.
__device__ __forceinline__ void forget(uint4& p) { asm volatile("" : "+v"(p.x), "+v"(p.y), "+v"(p.z), "+v"(p.w)); }

// Eight elements of the weight from element first + c on (first: the same in the
// workgroup).
__device__ __forceinline__ void load_weight(const void* weight, bool f32, int first, unsigned c, float (&w)[8]) {
  if (f32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(weight) + first + c);
    const float4 a = p[0], b = p[1];
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  } else {
    widen(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(weight) + first + c), w);
  }
}

// The row's sum (or maximum) over its THREADS threads; lds: one float a wave
// of the row, not in use by an earlier reduction that a thread may still read.
template <int THREADS, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* lds) {
  v = MAX ? wave_max(v) : wave_sum(v);
  if constexpr (THREADS > 64) {
    constexpr int W = THREADS / 64;
    if ((threadIdx.x & 63) == 0) lds[(threadIdx.x % THREADS) >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = MAX ? fmaxf(v, lds[i]) : v + lds[i];
  }
  return v;
}

__device__ __forceinline__ uint2 encode8(float (&v)[8], const CodeScale& u) {
  if (__any(u.lift != 1.0f)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = lifted_value<false>(v[e], u);
  }
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = fast_quotient(v[e], u.d, u.r);
  return make_uint2(code_pack2<false, true>(q[2], q[3], code_pack2<false, false>(q[0], q[1], 0u)),
                    code_pack2<false, true>(q[6], q[7], code_pack2<false, false>(q[4], q[5], 0u)));
}

template <int THREADS, int VPT, int OUT>
__global__ __launch_bounds__(THREADS > kThreads ? THREADS : kThreads) void rmsnorm_kernel(NormArgs a) {
  constexpr int kRows = THREADS < kThreads ? kThreads / THREADS : 1;  // of a workgroup
  constexpr int W = THREADS / 64;
  __shared__ float lds[2 * W];
  const int t = threadIdx.x % THREADS;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
  if (r >= a.rows) return;  // (a whole wave; rows of more than one wave have a workgroup to themselves)

  uint4 x[VPT], res[VPT];
  float w[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = ((int64_t)i * THREADS + t) * 8;
    x[i] = res[i] = make_uint4(0u, 0u, 0u, 0u);
    if (c < a.cols) {
      x[i] = read_once(a.x + r * a.ldx + c);
      if (a.residual) res[i] = read_once(a.residual + r * a.ldr + c);
    }
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = ((int64_t)i * THREADS + t) * 8;
    if (c < a.cols) {
      load_weight(a.weight, a.weight_f32 != 0, i * THREADS * 8, t * 8u, w[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[i][e] = 0.0f;
    }
  }
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    float v[8];
    widen(x[i], v);
    if (a.residual) {
      float q[8];
      widen(res[i], q);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += q[e];
      x[i] = narrow(v);
      widen(x[i], v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(v[e], v[e], sum);
  }
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = ((int64_t)i * THREADS + t) * 8;
      if (c < a.cols) write_once(a.h + r * a.ldh + c, x[i]);
    }
  }
  const float rstd = 1.0f / sqrtf(row_reduce<THREADS, false>(sum, lds) / (float)a.cols + a.eps);
  if (t == 0) a.rstd[r] = rstd;

  CodeScale u{};
  if constexpr (OUT == kNormRow) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float v[8];
      widen(x[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[e] * rstd * w[i][e]));
    }
    u = code_scale<false>(row_reduce<THREADS, true>(m, lds + W), a.pow2 != 0);
    if (t == 0) a.scales[r] = u.s;
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = ((int64_t)i * THREADS + t) * 8;
    float v[8];
    widen(x[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * rstd * w[i][e];
    if constexpr (OUT == kNormBlock) {
      float m = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[e]));
      u = code_scale<false>(row16_max(m), a.pow2 != 0);
      if ((t & 15) == 0 && c < a.cols) a.scales[(c >> 7) * a.rows + r] = u.s;
    }
    if (c < a.cols) {
      if constexpr (OUT == kNormBf16)
        *reinterpret_cast<uint4*>(a.y + r * a.ldy + c) = narrow(v);
      else
        *reinterpret_cast<uint2*>(a.codes + r * a.ldc + c) = encode8(v, u);
    }
  }
}

// Backward pass.  With xhat = h rstd and g = dy w,
//   dx = dres + rstd (g - xhat mean(g xhat)),   dw = sum over rows of dy xhat.
// dx is the gradient of x and of the residual alike.  8 bytes an element (dy,
// h, dres read, dx written; 6 without dres): a walker of THREADS threads takes
// rows walker, walker + walkers, ..., each held in registers, and keeps its part of
// dw there too; a workgroup's parts (four walkers of one wave meet in LDS) go to a
// workspace and a second kernel adds them in order, so the sum is the same on
// every run.  The loads of the next row are in flight while a row is worked on.
// 16384 x 4096 94 us (5.7 TB/s) with 512 workgroups; with 1024 110 us: their parts
// of dw are as many bytes as an eighth of the rows.  Up to 512 rows every row has a
// workgroup, and its part of dw costs as many bytes again as the row (512 x 4096 12.6 us).
template <int THREADS, int VPT>
__global__ __launch_bounds__(THREADS > kThreads ? THREADS : kThreads) void rmsnorm_backward_kernel(NormBackwardArgs a) {
  constexpr int kWalkers = THREADS < kThreads ? kThreads / THREADS : 1;  // of a workgroup
  constexpr int W = THREADS / 64;
  // registers: rows of more than 8192 elements leave no room for the next row and
  // for the weight, which is read again from L2 for every row
  constexpr bool kNext = THREADS <= 512, kHoldWeight = THREADS <= 512;
  __shared__ float lds[2][W];
  const int t = threadIdx.x % THREADS;
  const int64_t walkers = (int64_t)gridDim.x * kWalkers;
  const int64_t walker = (int64_t)blockIdx.x * kWalkers + threadIdx.x / THREADS;
  float held[kHoldWeight ? VPT : 1][8], dw[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = ((int64_t)i * THREADS + t) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
    if constexpr (kHoldWeight) {
#pragma unroll
      for (int e = 0; e < 8; ++e) held[i][e] = 0.0f;
      if (c < a.cols) load_weight(a.weight, a.weight_f32 != 0, i * THREADS * 8, t * 8u, held[i]);
    }
  }
  auto weight = [&](int i, float (&w)[8]) {
    const int64_t c = ((int64_t)i * THREADS + t) * 8;
    if constexpr (kHoldWeight) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = held[i][e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = 0.0f;
      // (loaded again for either pass of a row: kept between them it takes VPT x 8 registers)
      int first = i * THREADS * 8;
      asm volatile("" : "+s"(first));
      if (c < a.cols) load_weight(a.weight, a.weight_f32 != 0, first, t * 8u, w);
    }
  };
  uint4 dy[kNext ? 2 : 1][VPT], h[kNext ? 2 : 1][VPT], dres[kNext ? 2 : 1][VPT];
  auto fetch = [&](int64_t r, uint4 (&dy)[VPT], uint4 (&h)[VPT], uint4 (&dres)[VPT]) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = ((int64_t)i * THREADS + t) * 8;
      dy[i] = h[i] = dres[i] = make_uint4(0u, 0u, 0u, 0u);
      if (c < a.cols) {
        dy[i] = read_once(a.dy + r * a.lddy + c);
        h[i] = read_once(a.h + r * a.ldh + c);
        if (a.dres) dres[i] = read_once(a.dres + r * a.ldres + c);
      }
    }
  };
  // one row, held in dy, h and dres; turn: the row's part of lds (two in turn,
  // so that one barrier a row is enough)
  auto row = [&](int64_t r, int turn, uint4 (&dy)[VPT], uint4 (&h)[VPT], uint4 (&dres)[VPT]) {
    const float rstd = a.rstd[r];
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float d[8], x[8], w[8];
      widen(dy[i], d);
      widen(h[i], x);
      weight(i, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xhat = x[e] * rstd;
        dot = __builtin_fmaf(d[e] * w[e], xhat, dot);
        dw[i][e] = __builtin_fmaf(d[e], xhat, dw[i][e]);
      }
      forget(dy[i]);
      forget(h[i]);
      if constexpr (!kHoldWeight) {
        // the sums are formed here: moved past the next pieces' loads they keep the fp32
        // form of every piece, and rows of more than 16384 elements spill (4096 x 32768
        // 435 us, so 213)
        asm volatile("" : "+v"(dot));
#pragma unroll
        for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(dw[i][e]));
      }
    }
    const float mean = row_reduce<THREADS, false>(dot, lds[turn]) / (float)a.cols;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = ((int64_t)i * THREADS + t) * 8;
      float d[8], x[8], q[8], w[8];
      widen(dy[i], d);
      widen(h[i], x);
      widen(dres[i], q);
      weight(i, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float g = __builtin_fmaf(-(x[e] * rstd), mean, d[e] * w[e]);
        d[e] = __builtin_fmaf(rstd, g, q[e]);
      }
      if (c < a.cols) write_once(a.dx + r * a.lddx + c, narrow(d));
    }
  };
  if constexpr (kNext) {
    int64_t r = walker;
    if (r < a.rows) fetch(r, dy[0], h[0], dres[0]);
    for (; r < a.rows; r += 2 * walkers) {
      const bool second = r + walkers < a.rows, third = r + 2 * walkers < a.rows;
      if (second) fetch(r + walkers, dy[1], h[1], dres[1]);
      row(r, 0, dy[0], h[0], dres[0]);
      if (!second) break;
      if (third) fetch(r + 2 * walkers, dy[0], h[0], dres[0]);
      row(r + walkers, 1, dy[1], h[1], dres[1]);
    }
  } else {
    int turn = 0;
    for (int64_t r = walker; r < a.rows; r += walkers, turn ^= 1) {
      fetch(r, dy[0], h[0], dres[0]);
      row(r, turn, dy[0], h[0], dres[0]);
    }
  }
  if constexpr (kWalkers > 1) {
    __shared__ float parts[kWalkers - 1][VPT][8][64];
    const int wave = threadIdx.x >> 6;
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) parts[wave - 1][i][e][t] = dw[i][e];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < kWalkers - 1; ++w)
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] += parts[w][i][e][t];
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = ((int64_t)i * THREADS + t) * 8;
    if (c < a.cols) {
      float4* p = reinterpret_cast<float4*>(a.partials + blockIdx.x * a.cols + c);
      p[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
      p[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
    }
  }
}

// dweight from the workgroups' parts: a workgroup takes 64 columns, its sixteen
// waves every sixteenth part each, eight loads in flight; LDS joins the waves
// in order.
constexpr int kReduceWaves = 16, kReduceDepth = 8;

__global__ __launch_bounds__(kReduceWaves * 64) void norm_weight_kernel(const float* partials, int64_t groups,
                                                                        int64_t cols, float* dweight) {
  __shared__ float lds[kReduceWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (c < cols) {
    for (int64_t g0 = wave; g0 < groups; g0 += kReduceWaves * kReduceDepth) {
      float v[kReduceDepth];
#pragma unroll
      for (int j = 0; j < kReduceDepth; ++j) {
        const int64_t g = g0 + (int64_t)kReduceWaves * j;
        v[j] = g < groups ? partials[g * cols + c] : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < kReduceDepth; ++j) sum += v[j];
    }
  }
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && c < cols) {
#pragma unroll
    for (int w = 1; w < kReduceWaves; ++w) sum += lds[w][lane];
    dweight[c] = sum;
  }
}

// f(THREADS, VPT) as integral constants: threads of a row and 16-byte pieces
// of each.  One wave a row up to 1024 elements (no barrier), four up to 6144,
// eight up to 8192, sixteen above.
template <typename F>
hipError_t with_shape(int64_t cols, F&& f) {
  using std::integral_constant;
  if (cols <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (cols <= 1024) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (cols <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (cols <= 4096) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (cols <= 6144) return f(integral_constant<int, 256>{}, integral_constant<int, 3>{});
  if (cols <= 8192) return f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  if (cols <= 16384) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  if (cols <= kMaxNormCols) return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
  return hipErrorInvalidValue;
}

template <int OUT>
hipError_t launch_out(const NormArgs& a, hipStream_t s) {
  return with_shape(a.cols, [&](auto threads, auto vpt) {
    constexpr int T = decltype(threads)::value, V = decltype(vpt)::value;
    constexpr int block = T > kThreads ? T : kThreads, rows = T < kThreads ? kThreads / T : 1;
    const int64_t grid = (a.rows + rows - 1) / rows;
    rmsnorm_kernel<T, V, OUT><<<dim3((unsigned)grid), block, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace norm_detail

using namespace norm_detail;

hipError_t launch_rmsnorm(const NormArgs& a, NormOut out, hipStream_t s) {
  switch (out) {
    case kNormBf16: return launch_out<kNormBf16>(a, s);
    case kNormRow: return launch_out<kNormRow>(a, s);
    case kNormBlock: return launch_out<kNormBlock>(a, s);
    default: return hipErrorInvalidValue;
  }
}

int64_t norm_backward_groups(int64_t rows, int64_t cols) {
  // two workgroups of 256 threads a CU (16384 x 1024 29.0 us, with 1024 of them
  // 35.5; 16384 x 4096 above), one of 512 or 1024 (8192 x 8192 97.9, with two 102)
  const int64_t most = cols <= 6144 ? 512 : 256, ready = cols <= 1024 ? (rows + 3) / 4 : rows;
  return ready < most ? ready : most;
}

hipError_t launch_rmsnorm_backward(const NormBackwardArgs& a, hipStream_t s) {
  const int64_t groups = norm_backward_groups(a.rows, a.cols);
  const hipError_t e = with_shape(a.cols, [&](auto threads, auto vpt) {
    constexpr int T = decltype(threads)::value, V = decltype(vpt)::value;
    rmsnorm_backward_kernel<T, V><<<dim3((unsigned)groups), T > kThreads ? T : kThreads, 0, s>>>(a);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  norm_weight_kernel<<<dim3((unsigned)((a.cols + 63) / 64)), kReduceWaves * 64, 0, s>>>(a.partials, groups, a.cols,
                                                                                       a.dweight);
  return hipGetLastError();
}

}  // namespace fp8q
