// Log-probabilities of the taken tokens, entropies, and the k most probable alternatives of
// each row of logits, on gfx950.
//
// With z = x / temperature, lse = log sum exp(z): logp = z_token - lse, entropy = lse - sum p
// z, and the k largest logits' indices with their z - lse, in descending order, equal logits
// by index.  A logit of -inf is no alternative; where a row has fewer than k others, the
// places left over get the index -1 and -inf.
//
// Bound by HBM: the logits read once.  The pass that takes the running maximum and sums leaves
// the largest logit of every slot (a thread's elements, or those of 64 in a row that is shared by
// workgroups).  The slots fall into 64 or 256 groups; the k-th largest of the groups' maxima, cut to 16
// bits, is at most the row's k-th largest logit (k elements are as large): a bound that few elements pass, all of them
// in slots whose maximum passes.  Those slots are read again (from the caches), and what passes is
// ranked by counting.  Where more pass than LDS has room for (logits that are all equal, say),
// the k largest are taken one after the other from the row: slower, and right for any row.
#include "logits.h"
#include "rollout.h"

namespace fp8q {

namespace top_detail {

using namespace logits_detail;

// A logit's place in the order of the alternatives: larger logits first, then lower indices;
// 0 for none.  (-0 counts as 0.)
typedef uint64_t Key;
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ Key key_of(float x, uint32_t index) {
  return x > kNegInf ? (Key)ordered(x) << 32 | (uint32_t)~index : 0;  // (NaN: none)
}
__device__ __forceinline__ float logit_of(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t index_of(Key k) { return ~(uint32_t)k; }

// z - lse of a logit, from the row's sums.
struct LogProb {
  Exponent exponent;
  float c, m, log_s;
  __device__ __forceinline__ LogProb(const Sums& sums, float c_) : exponent(c_, sums.m), c(c_), m(sums.m), log_s(logf(sums.s)) {}
  __device__ __forceinline__ float operator()(float x) const {
    const float u = exponent.c == c ? exponent(x) : (x - m) * c;
    return __builtin_fmaf(u, kLn2, -log_s);
  }
};
__device__ __forceinline__ float entropy_of(const Sums& sums) { return logf(sums.s) - kLn2 * (sums.q / sums.s); }

__device__ __forceinline__ bool in_vocabulary(const TopArgs& a, int64_t token) { return token >= 0 && token < a.V; }

// What a row gets: its token's results, and the alternative at place i.
__device__ __forceinline__ void put_token(const TopArgs& a, int64_t row, const Sums& sums, float x) {
  a.logp[row] = LogProb(sums, a.inv_temperature * kLog2e)(x);
  a.entropy[row] = entropy_of(sums);
}
__device__ __forceinline__ void put_alternative(const TopArgs& a, int64_t row, int i, Key k, const LogProb& lp) {
  a.ids[row * a.k + i] = k ? (int64_t)index_of(k) : -1;
  a.top[row * a.k + i] = k ? lp(logit_of(k)) : kNegInf;
}
// A row whose token is outside the vocabulary.
template <int THREADS>
__device__ __forceinline__ void put_nothing(const TopArgs& a, int64_t row) {
  const int t = threadIdx.x;
  if (t < a.k) {
    a.ids[row * a.k + t] = -1;
    a.top[row * a.k + t] = 0.0f;
  }
  if (t == 0) a.logp[row] = a.entropy[row] = 0.0f;
}

// The maximum of 64-bit keys over a wave.
__device__ __forceinline__ Key wave_max_key(Key k) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const Key o = (Key)(uint32_t)__shfl_xor((int)(k >> 32), d, 64) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)k, d, 64);
    k = o > k ? o : k;
  }
  return k;
}

constexpr int kCandidates = 1024;

// LDS of the selection among SLOTS slots.
template <int THREADS, int SLOTS>
struct Selection {
  float maxima[THREADS];
  uint16_t slots[SLOTS];
  Key keys[kCandidates];
  Key wave_keys[THREADS / 64];
  int selected, candidates;
};

// At most the k-th largest of the N values that each of a wave's 64 lanes holds (k <= 64): its
// upper 16 bits in the logits' order, bit by bit from the top, each by counting the values that reach it.
template <int N>
__device__ __forceinline__ float bound_of_wave(const float (&v)[N], int k) {
  uint32_t o[N], b = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = ordered(v[i]) >> 16;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t c = b | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += (int)__popcll(__ballot(o[i] >= c));
    if (n >= k) b = c;
  }
  // (0x7f: those of -inf and NaN)
  return b <= 0x7f ? kNegInf : logit_of((Key)(b << 16) << 32);
}

// The bound of a row whose slots' maxima are `most` of each thread, in groups by t % 64, or by t
// % 256 for a large k, where 64 groups let through a multiple of k (about 64 log(64 / (64 - k))
// elements: 64 x 131072 bf16, k = 64, 54 us, with 256 groups 22; k = 5 15.5 and 16.2).
template <int THREADS, int SLOTS>
__device__ __forceinline__ float bound_of(Selection<THREADS, SLOTS>& s, float most, int k) {
  const int t = threadIdx.x, lane = t & 63;
  s.maxima[t] = most;
  if (t == 0) s.selected = s.candidates = 0;
  __syncthreads();
  float group[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    group[i] = s.maxima[i * 64 + lane];
#pragma unroll
    for (int w = 4 + i; w < THREADS / 64; w += 4) group[i] = fmaxf(group[i], s.maxima[w * 64 + lane]);
  }
  if (k > 24) return bound_of_wave(group, k);
  const float all[1] = {fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3]))};
  return bound_of_wave(all, k);
}

template <int THREADS, int SLOTS>
__device__ __forceinline__ void select_slot(Selection<THREADS, SLOTS>& s, int slot, float most, float bound) {
  if (most >= bound && most > kNegInf)
    s.slots[__hip_atomic_fetch_add(&s.selected, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)] = (uint16_t)slot;
}

// The k largest elements of a row, into the first k of s.keys, in order (0: none), after
// select_slot for every slot.  piece(slot, i): piece i, of `per`, of a slot, or -1; `edge`: this
// thread's single element, or -1.
template <bool F32, int THREADS, int SLOTS, typename Slot>
__device__ __forceinline__ void select_top(Selection<THREADS, SLOTS>& s, const Row<F32>& x, int edge, float bound, int k,
                                           int per, Slot&& piece) {
  using P = Piece<F32>;
  constexpr int W = THREADS / 64;
  const int t = threadIdx.x, lane = t & 63;
  __syncthreads();
  auto offer = [&](float v, int index) {
    if (v >= bound && v > kNegInf) {
      const int n = __hip_atomic_fetch_add(&s.candidates, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      if (n < kCandidates) s.keys[n] = key_of(v, (uint32_t)index);
    }
  };
  auto load = [&](int j) { return *reinterpret_cast<const uint4*>(x.base + x.head * P::kSize + (int64_t)j * 16); };
  auto each = [&](int j, const uint4& p, auto&& f) {
    float v[P::kN];
    P::widen(p, v);
#pragma unroll
    for (int e = 0; e < P::kN; ++e) f(v[e], x.head + j * P::kN + e);
  };
  // (in any order: the keys are all different)
  const int work = s.selected * per;
  for (int q = t; q < work; q += THREADS) {
    const int from = q / per, j = piece(s.slots[from], q - from * per);
    if (j >= 0) each(j, load(j), offer);
  }
  if (edge >= 0) offer(P::load(x.base, edge), edge);
  __syncthreads();
  const int n = s.candidates;
  if (n <= kCandidates) {
    constexpr int kMine = (kCandidates + THREADS - 1) / THREADS;
    Key mine[kMine];
    int rank[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = t + i * THREADS;
      mine[i] = at < n ? s.keys[at] : 0;
      rank[i] = 0;
    }
    if ((t & ~63) < n) {  // (waves with a candidate)
      for (int j = 0; j < n; ++j) {
        const Key o = s.keys[j];
#pragma unroll
        for (int i = 0; i < kMine; ++i) rank[i] += o > mine[i] ? 1 : 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if (t + i * THREADS < n && rank[i] < k) s.keys[rank[i]] = mine[i];
    if (t >= n && t < k) s.keys[t] = 0;
    __syncthreads();
    return;
  }
  // too many: the largest below the one before, k times
  Key before = ~(Key)0;
  for (int i = 0; i < k; ++i) {
    Key best = 0;
    auto meet = [&](float v, int index) {
      const Key o = key_of(v, (uint32_t)index);
      best = o < before && o > best ? o : best;
    };
    for (int j = t; j < x.full; j += THREADS) each(j, load(j), meet);
    if (edge >= 0) meet(P::load(x.base, edge), edge);
    best = wave_max_key(best);
    if (lane == 0) s.wave_keys[t >> 6] = best;
    __syncthreads();
    best = s.wave_keys[0];
#pragma unroll
    for (int w = 1; w < W; ++w) best = s.wave_keys[w] > best ? s.wave_keys[w] : best;
    before = best;
    __syncthreads();
    if (t == 0) s.keys[i] = best;
  }
  __syncthreads();
}

// The sums of pieces first + t + i THREADS below last and of this thread's edge; NV in flight.
// Chunks that are nothing but padding for the whole workgroup are left out (64 x 131072 bf16 15.1
// -> 13.5 us of kernels, 16.8 -> 15.2 a pass, 2048 x 8000 fp32 22.2 -> 20.0 a pass; where none is, up to 2% for
// the test; workgroups of 1024 have rows that fill them and lost as much).
template <bool F32, int THREADS, int NV>
__device__ __forceinline__ Sums own_sums(const Row<F32>& x, int first, int last, int edge, float c) {
  using P = Piece<F32>;
  constexpr int kChunk = NV % 4 == 0 ? 4 : NV;
  Sums sums{kNegInf, 0.0f, 0.0f};
  for (int j0 = first; j0 < last; j0 += NV * THREADS) {
    uint4 held[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) held[i] = x.piece(j0 + i * THREADS, last, threadIdx.x);
#pragma unroll
    for (int i = 0; i < NV; i += kChunk) {
      if (THREADS < 1024 && j0 + i * THREADS >= last) break;
      add_pieces<F32, kChunk>(held + i, c, sums);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (edge >= 0) sums = join(sums, single(P::load(x.base, edge), c), c);
  return sums;
}

// One workgroup a row.
template <bool F32, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void top_row_kernel(TopArgs a) {
  constexpr int W = THREADS / 64;
  __shared__ Selection<THREADS, THREADS> selection;
  __shared__ Sums parts[W];
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x, token = a.tokens[row];
  if (!in_vocabulary(a, token)) return put_nothing<THREADS>(a, row);  // the whole workgroup
  const float c = a.inv_temperature * kLog2e;
  const Row<F32> x(a.logits, a.ld, row, a.V);
  const float mine = Piece<F32>::load(x.base, token);
  const int edge = x.edge(t);
  Sums sums = own_sums<F32, THREADS, NV>(x, 0, x.full, edge, c);
  const float most = sums.m;
  sums = wave_join(sums, c);
  if ((t & 63) == 0) parts[t >> 6] = sums;
  const float bound = bound_of(selection, most, a.k);
  select_slot(selection, t, most, bound);
  select_top(selection, x, edge, bound, a.k, (x.full + THREADS - 1) / THREADS, [&](int slot, int i) {
    const int j = slot + i * THREADS;
    return j < x.full ? j : -1;
  });
  sums = wave_join<W>(parts[t & (W - 1)], c);
  if (t < 64) {
    const LogProb lp(sums, c);
    if (t < a.k) put_alternative(a, row, t, selection.keys[t], lp);
    if (t == 0) put_token(a, row, sums, mine);
  }
}

// Few rows: workgroup (part, row) takes the pieces j with j / per == part, and part 0 the row's
// edges, and leaves sums and the maxima of 64 slots, the pieces and threads with equal t % 64;
// a second kernel joins the sums and selects.
constexpr int kSplitThreads = 256;

// The workspace: the parts' sums and the token's logit, [T][kLossParts] of four floats, then
// the slots' maxima, [T][kLossParts][64].
__device__ __forceinline__ float4* part_sums(const TopArgs& a, int64_t row) {
  return reinterpret_cast<float4*>(a.workspace) + row * kLossParts;
}
__device__ __forceinline__ float* part_maxima(const TopArgs& a, int64_t row) {
  return reinterpret_cast<float*>(a.workspace + a.T * kLossParts * 16) + row * kLossParts * 64;
}

template <bool F32>
__global__ __launch_bounds__(kSplitThreads) void top_part_kernel(TopArgs a, int per) {
  constexpr int W = kSplitThreads / 64;
  __shared__ float maxima[kSplitThreads];
  __shared__ Sums parts[W];
  const int t = threadIdx.x;
  const int64_t part = blockIdx.x, row = blockIdx.y, token = a.tokens[row];
  if (!in_vocabulary(a, token)) return;
  const float c = a.inv_temperature * kLog2e;
  const Row<F32> x(a.logits, a.ld, row, a.V);
  const int first = (int)part * per, last = first + per < x.full ? first + per : x.full;
  const int edge = part == 0 ? x.edge(t) : -1;
  Sums sums = own_sums<F32, kSplitThreads, 8>(x, first, last, edge, c);
  maxima[t] = sums.m;
  sums = wave_join(sums, c);
  if ((t & 63) == 0) parts[t >> 6] = sums;
  __syncthreads();
  if (t >= 64) return;
  float most = maxima[t];
#pragma unroll
  for (int w = 1; w < W; ++w) most = fmaxf(most, maxima[w * 64 + t]);
  part_maxima(a, row)[part * 64 + t] = most;
  sums = wave_join<W>(parts[t & (W - 1)], c);
  if (t == 0)
    part_sums(a, row)[part] = make_float4(sums.m, sums.s, sums.q, part == 0 ? Piece<F32>::load(x.base, token) : 0.0f);
}

template <bool F32>
__global__ __launch_bounds__(kSplitThreads) void top_join_kernel(TopArgs a, int per, int parts) {
  constexpr int kSlots = kLossParts * 64, kMine = kSlots / kSplitThreads;
  __shared__ Selection<kSplitThreads, kSlots> selection;
  const int t = threadIdx.x, lane = t & 63;
  const int64_t row = blockIdx.x;
  // (the loads go out together with the token's; a row that is not read has left nothing here)
  const int64_t token = a.tokens[row];
  const float c = a.inv_temperature * kLog2e;
  const Row<F32> x(a.logits, a.ld, row, a.V);
  const float* const maxima = part_maxima(a, row);
  float own[kMine], most = kNegInf;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    own[i] = t + i * kSplitThreads < parts * 64 ? maxima[t + i * kSplitThreads] : kNegInf;
    most = fmaxf(most, own[i]);
  }
  float4 p = make_float4(kNegInf, 0.0f, 0.0f, 0.0f);
  if (lane < parts) p = part_sums(a, row)[lane];
  const float mine = part_sums(a, row)[0].w;
  if (!in_vocabulary(a, token)) return put_nothing<kSplitThreads>(a, row);
  const float bound = bound_of(selection, most, a.k);
#pragma unroll
  for (int i = 0; i < kMine; ++i) select_slot(selection, t + i * kSplitThreads, own[i], bound);
  select_top(selection, x, x.edge(t), bound, a.k, (per + 63) / 64, [&](int slot, int i) {
    const int first = (slot >> 6) * per, last = first + per < x.full ? first + per : x.full;
    const int j = first + (slot & 63) + i * 64;
    return j < last ? j : -1;
  });
  if (t < 64) {
    const Sums sums = wave_join(Sums{p.x, p.y, p.z}, c);
    const LogProb lp(sums, c);
    if (t < a.k) put_alternative(a, row, t, selection.keys[t], lp);
    if (t == 0) put_token(a, row, sums, mine);
  }
}

// Pieces of each of the workgroups that share a row, and their number.
inline int split_parts(int64_t T, int64_t pieces, int& per) {
  int64_t parts = (1024 + T - 1) / T;
  const int64_t most = (pieces + kSplitThreads * 4 - 1) / (kSplitThreads * 4);
  if (parts > most) parts = most;
  if (parts > kLossParts) parts = kLossParts;
  if (parts < 1) parts = 1;
  per = (int)((pieces + parts - 1) / parts);
  return (int)parts;
}

// Whether rows are split over workgroups: as the log-probabilities alone.
inline bool split_rows(int64_t T, int64_t V) {
  return T < kLossSplitRows && (double)V * (6.2e-5 - 5.4e-7 * (double)T) > 3.0;
}

template <bool F32>
hipError_t launch_top(const TopArgs& a, hipStream_t s) {
  const int64_t pieces = a.V / Piece<F32>::kN;
  if (split_rows(a.T, a.V)) {
    int per;
    const int parts = split_parts(a.T, pieces, per);
    top_part_kernel<F32><<<dim3((unsigned)parts, (unsigned)a.T), kSplitThreads, 0, s>>>(a, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    top_join_kernel<F32><<<dim3((unsigned)a.T), kSplitThreads, 0, s>>>(a, per, parts);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)a.T);
  if (pieces <= 4 * 256)
    top_row_kernel<F32, 256, 4><<<grid, 256, 0, s>>>(a);
  else if (pieces <= 8 * 512)
    top_row_kernel<F32, 512, 8><<<grid, 512, 0, s>>>(a);
  else
    top_row_kernel<F32, 1024, 8><<<grid, 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace top_detail

using namespace top_detail;

int64_t top_logprobs_workspace(int64_t T, int64_t V) {
  return split_rows(T, V) ? T * kLossParts * (16 + 4 * 64) : 0;
}

hipError_t launch_top_logprobs(const TopArgs& a, hipStream_t s) {
  return a.f32 ? launch_top<true>(a, s) : launch_top<false>(a, s);
}

}  // namespace fp8q
