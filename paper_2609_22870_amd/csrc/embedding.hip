// The embedding table's rows for a batch of tokens, and the table's gradient, on gfx950.
//
//   y[t] = scale w[token_t],    dw[v] = scale sum over token_t = v of dy[t]
//
// A token outside 0 .. V-1 (padding) gives a row of zeros and takes no part in the gradient.
//
// The gradient sums each row in the order of t, in fp32, so that every run gives the same
// bits: the tokens are sorted (stably: by token, then by t), the sorted positions are cut into
// chunks of kChunk, and a workgroup adds up the rows of dy of one chunk, over a band of columns,
// run by run of equal tokens.  A run inside a chunk goes to the table at once; one that crosses
// chunks leaves a sum per chunk in the workspace, and a second kernel adds those in order.
// The rows of tokens that do not occur are filled with zeros by the same launch (a bitmap of
// those that do comes with the sort), which is most of what a whole gradient costs: bound by
// HBM, V C elements written and T C read.
#include "device_common.h"
#include "rollout.h"

namespace fp8q {

namespace embedding_detail {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{lo, hi}), v2bf));
}

// Eight elements as fp32 and back.
struct Eight {
  float v[8];
  __device__ __forceinline__ void widen(const v4u& p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = bf16_lo(p[e]);
      v[2 * e + 1] = bf16_hi(p[e]);
    }
  }
  __device__ __forceinline__ v4u narrow() const {
    return v4u{bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7])};
  }
};

constexpr int kThreads = 256, kBand = kThreads * 8;  // a workgroup's columns

// Four tokens a workgroup, eight columns a thread, all four rows' loads in flight.
constexpr int kLookupRows = 4;
template <bool F32>
__global__ __launch_bounds__(kThreads) void embedding_kernel(EmbeddingArgs a, int bands) {
  const int64_t t0 = (int64_t)(blockIdx.x / bands) * kLookupRows;
  const int64_t c = (int64_t)(blockIdx.x % bands) * kBand + threadIdx.x * 8;
  if (c >= a.C) return;
  v4u p[kLookupRows], q[kLookupRows];
#pragma unroll
  for (int i = 0; i < kLookupRows; ++i) {
    const int64_t token = t0 + i < a.T ? a.tokens[t0 + i] : -1;
    p[i] = q[i] = v4u{0, 0, 0, 0};
    if (token < 0 || token >= a.V) continue;
    if constexpr (F32) {
      const v4u* const from = reinterpret_cast<const v4u*>(static_cast<const float*>(a.weight) + token * a.ldw + c);
      p[i] = from[0];
      q[i] = from[1];
    } else {
      p[i] = *reinterpret_cast<const v4u*>(static_cast<const uint16_t*>(a.weight) + token * a.ldw + c);
    }
  }
#pragma unroll
  for (int i = 0; i < kLookupRows; ++i) {
    if (t0 + i >= a.T) break;
    Eight x;
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x.v[e] = __uint_as_float(p[i][e]);
        x.v[4 + e] = __uint_as_float(q[i][e]);
      }
    } else {
      x.widen(p[i]);
    }
    const int64_t token = a.tokens[t0 + i];
    const bool live = token >= 0 && token < a.V;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = live ? x.v[e] * a.scale : 0.0f;
    *reinterpret_cast<v4u*>(a.y + (t0 + i) * a.ldy + c) = x.narrow();
  }
}

// ---- the sort -----------------------------------------------------------------------------
//
// Radix sort by the token, least significant digit first; tokens outside the vocabulary take
// the key V.  A wave ranks 64 keys at a time, in order: the lanes with its digit are found by
// a ballot per bit, the count of those before them in the wave from a counter in LDS.

// The lanes whose BITS-bit digit is this lane's (of those that are live).
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool live) {
  uint64_t m = __ballot(live);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const bool one = digit >> b & 1;
    const uint64_t o = __ballot(one);
    m &= one ? o : ~o;
  }
  return m;
}

// A wave's LDS operations before this point come before those after it, for all its lanes.
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// This lane's place among its wave's keys of the same digit so far (counter: the wave's, of
// this digit), and the counter moved on.
template <int BITS>
__device__ __forceinline__ uint32_t rank_in_wave(uint32_t digit, bool live, uint32_t* counters) {
  const int lane = threadIdx.x & 63;
  const uint64_t m = same_digit<BITS>(digit, live);
  const uint64_t below = m & (((uint64_t)1 << lane) - 1);
  uint32_t before = 0;
  if (live) before = counters[digit];
  in_order();
  if (live && below == 0) counters[digit] = before + (uint32_t)__popcll(m);
  in_order();
  return before + (uint32_t)__popcll(below);
}

// Exclusive prefix sums of n counters in LDS by THREADS threads, n a multiple of THREADS.
template <int THREADS>
__device__ __forceinline__ void prefix_sums(uint32_t* counters, int n, uint32_t* wave_sums) {
  const int t = threadIdx.x, lane = t & 63, per = n / THREADS;
  uint32_t sum = 0;
  for (int i = 0; i < per; ++i) sum += counters[t * per + i];
  uint32_t scan = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(scan, d, 64);
    if (lane >= d) scan += o;
  }
  if (lane == 63) wave_sums[t >> 6] = scan;
  __syncthreads();
  uint32_t base = scan - sum;
  for (int w = 0; w < t >> 6; ++w) base += wave_sums[w];
  for (int i = 0; i < per; ++i) {
    const uint32_t c = counters[t * per + i];
    counters[t * per + i] = base;
    base += c;
  }
  __syncthreads();
}

__device__ __forceinline__ uint32_t key_of(int64_t token, int64_t V) {
  return token >= 0 && token < V ? (uint32_t)token : (uint32_t)V;
}

// Up to kSortMost tokens in one workgroup: a word holds key and t together (kPosBits for
// t), so the pass that a key makes is one word through LDS.  Wave w has the words from w
// 64 rounds on, so that its rounds go in order.
constexpr int kSortThreads = 1024, kSortWaves = 16, kSortRounds = 16, kPosBits = 14;
constexpr int64_t kSortMost = 16384;
constexpr int kDigit = 6;  // bits a pass

__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(const int64_t* tokens, int T, int64_t V, int key_bits,
                                                                  uint32_t* keys, uint32_t* positions,
                                                                  uint32_t* bitmap) {
  __shared__ uint32_t words[kSortMost];
  __shared__ uint32_t counters[kSortWaves << kDigit], sums[kSortWaves];  // [digit][wave]
  __shared__ uint32_t mine_lds[kSortWaves][1 << kDigit];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int rounds = (T + kSortThreads - 1) / kSortThreads, first = wave * rounds * 64 + lane;
  for (int64_t i = t; i < (V + 31) / 32; i += kSortThreads) bitmap[i] = 0;
  uint32_t w[kSortRounds], rank[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = first + r * 64;
    w[r] = 0xffffffffu;
    if (r < rounds && i < T) w[r] = key_of(tokens[i], V) << kPosBits | (uint32_t)i;
  }
  uint32_t* const mine = mine_lds[wave];
  for (int shift = 0; shift < key_bits; shift += kDigit) {
    mine[lane] = 0;
    in_order();
    auto digit_of = [&](uint32_t x) { return x >> (kPosBits + shift) & ((1u << kDigit) - 1); };
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (r < rounds) rank[r] = rank_in_wave<kDigit>(digit_of(w[r]), first + r * 64 < T, mine);
    __syncthreads();
    counters[lane * kSortWaves + wave] = mine[lane];
    __syncthreads();
    prefix_sums<kSortThreads>(counters, kSortWaves << kDigit, sums);
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (r < rounds && first + r * 64 < T) words[counters[digit_of(w[r]) * kSortWaves + wave] + rank[r]] = w[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (r < rounds && first + r * 64 < T) w[r] = words[first + r * 64];
    __syncthreads();
  }
  // (the bitmap's zeros are in memory: a barrier waits for the workgroup's own stores)
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = first + r * 64;
    if (r < rounds && i < T) {
      const uint32_t key = w[r] >> kPosBits;
      keys[i] = key;
      positions[i] = w[r] & ((1u << kPosBits) - 1);
      if (key < (uint32_t)V && (i == 0 || words[i - 1] >> kPosBits != key))
        __hip_atomic_fetch_or(bitmap + (key >> 5), 1u << (key & 31), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
}

// More tokens: tiles of kTile in a workgroup each, a pass being three launches (the tiles'
// counts by digit, their prefix sums, the words to their places).  The first pass reads the tokens.
constexpr int kTileThreads = 256, kTileWaves = 4, kTileRounds = 16, kTile = kTileThreads * kTileRounds;
constexpr int kWideDigit = 8;

struct SortPass {
  const int64_t* tokens;  // of the first pass, else null
  const uint32_t *keys, *positions;
  uint32_t *keys_out, *positions_out;
  uint32_t* counts;  // [256][tiles]
  int64_t T, V;
  int tiles, shift;
  uint32_t* bitmap;  // of the last pass, else null
  __device__ __forceinline__ uint32_t key(int64_t i) const { return tokens ? key_of(tokens[i], V) : keys[i]; }
  __device__ __forceinline__ uint32_t digit(uint32_t k) const { return k >> shift & ((1u << kWideDigit) - 1); }
};

__global__ __launch_bounds__(kTileThreads) void sort_count_kernel(SortPass p) {
  __shared__ uint32_t counts[1 << kWideDigit];
  const int t = threadIdx.x;
  counts[t] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kTile + t;
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int64_t i = first + r * kTileThreads;
    if (i < p.T) __hip_atomic_fetch_add(counts + p.digit(p.key(i)), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  __syncthreads();
  p.counts[(int64_t)t * p.tiles + blockIdx.x] = counts[t];
  if (p.bitmap)
    for (int64_t i = first; i < (p.V + 31) / 32; i += (int64_t)gridDim.x * kTile)
      for (int r = 0; r < kTileRounds; ++r)
        if (i + r * kTileThreads < (p.V + 31) / 32) p.bitmap[i + r * kTileThreads] = 0;
}

// Exclusive prefix sums of n counts, by one workgroup.
__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(uint32_t* counts, int64_t n) {
  __shared__ uint32_t sums[kSortWaves];
  const int t = threadIdx.x, lane = t & 63;
  uint32_t carry = 0;
  constexpr int kPer = 8;
  for (int64_t first = 0; first < n; first += kSortThreads * kPer) {
    uint32_t v[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t at = first + t * kPer + i;
      v[i] = at < n ? counts[at] : 0;
      sum += v[i];
    }
    uint32_t scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = __shfl_up(scan, d, 64);
      if (lane >= d) scan += o;
    }
    if (lane == 63) sums[t >> 6] = scan;
    __syncthreads();
    uint32_t base = carry + scan - sum, all = 0;
    for (int w = 0; w < kSortWaves; ++w) {
      if (w < t >> 6) base += sums[w];
      all += sums[w];
    }
    carry += all;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int64_t at = first + t * kPer + i;
      if (at < n) counts[at] = base;
      base += v[i];
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(kTileThreads) void sort_move_kernel(SortPass p) {
  __shared__ uint32_t counters[kTileWaves][1 << kWideDigit];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t first = (int64_t)blockIdx.x * kTile + wave * (kTileRounds * 64) + lane;
  for (int d = lane; d < 1 << kWideDigit; d += 64) counters[wave][d] = 0;
  in_order();
  uint32_t key[kTileRounds], rank[kTileRounds];
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int64_t i = first + r * 64;
    key[r] = i < p.T ? p.key(i) : 0;
  }
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r)
    rank[r] = rank_in_wave<kWideDigit>(p.digit(key[r]), first + r * 64 < p.T, counters[wave]);
  __syncthreads();
  // each digit's waves, in order, after the digit's place for this tile
  uint32_t base = p.counts[(int64_t)t * p.tiles + blockIdx.x];
#pragma unroll
  for (int w = 0; w < kTileWaves; ++w) {
    const uint32_t c = counters[w][t];
    counters[w][t] = base;
    base += c;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int64_t i = first + r * 64;
    if (i >= p.T) continue;
    const uint32_t to = counters[wave][p.digit(key[r])] + rank[r];
    p.keys_out[to] = key[r];
    p.positions_out[to] = p.tokens ? (uint32_t)i : p.positions[i];
    if (p.bitmap && key[r] < (uint32_t)p.V)
      __hip_atomic_fetch_or(p.bitmap + (key[r] >> 5), 1u << (key[r] & 31), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// ---- the sums -----------------------------------------------------------------------------

struct Gradient {
  EmbeddingBackwardArgs a;
  const uint32_t *keys, *positions, *bitmap;
  float* partials;  // [chunks][2][C]: the sums of a run from the chunk before, and of one into the next
  int chunk;        // positions of a chunk
  int chunks, bands;
};

// Columns c .. c + 7 of row v of the table.
__device__ __forceinline__ void put_row(const EmbeddingBackwardArgs& a, uint32_t v, int64_t c, const Eight& sum) {
  Eight x;
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = sum.v[e] * a.scale;
  const int64_t at = (int64_t)v * a.ldw + c;
  if (a.f32) {
    v4u* const to = reinterpret_cast<v4u*>(static_cast<float*>(a.dweight) + at);
    v4u lo, hi;
    if (a.accumulate) {
      lo = to[0];
      hi = to[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x.v[e] += __uint_as_float(lo[e]);
        x.v[4 + e] += __uint_as_float(hi[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = __float_as_uint(x.v[e]);
      hi[e] = __float_as_uint(x.v[4 + e]);
    }
    __builtin_nontemporal_store(lo, to);
    __builtin_nontemporal_store(hi, to + 1);
  } else {
    v4u* const to = reinterpret_cast<v4u*>(static_cast<uint16_t*>(a.dweight) + at);
    if (a.accumulate) {
      Eight old;
      old.widen(*to);
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[e] += old.v[e];
    }
    __builtin_nontemporal_store(x.narrow(), to);
  }
}

// The first chunks * bands workgroups sum a chunk over a band of columns each; the others fill
// kFillRows rows of the table with zeros where no token names them.
constexpr int kFillRows = 8, kAhead = 8;  // rows of dy in flight

__global__ __launch_bounds__(kThreads) void embedding_sums_kernel(Gradient g) {
  const EmbeddingBackwardArgs& a = g.a;
  const unsigned sums = (unsigned)g.chunks * g.bands;
  const unsigned b = blockIdx.x < sums ? blockIdx.x : blockIdx.x - sums;
  const int64_t c = (int64_t)(b % g.bands) * kBand + threadIdx.x * 8;
  if (c >= a.C) return;
  if (blockIdx.x >= sums) {
    const int64_t v0 = (int64_t)(b / g.bands) * kFillRows;  // (a word of the bitmap has whole groups)
    const uint32_t used = g.bitmap[v0 >> 5] >> (v0 & 31);
    const v4u zero = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kFillRows; ++i) {
      if (v0 + i >= a.V || (used >> i & 1)) continue;
      const int64_t at = (v0 + i) * a.ldw + c;
      if (a.f32) {
        v4u* const to = reinterpret_cast<v4u*>(static_cast<float*>(a.dweight) + at);
        __builtin_nontemporal_store(zero, to);
        __builtin_nontemporal_store(zero, to + 1);
      } else {
        __builtin_nontemporal_store(zero, reinterpret_cast<v4u*>(static_cast<uint16_t*>(a.dweight) + at));
      }
    }
    return;
  }
  const int64_t first = (int64_t)(b / g.bands) * g.chunk, last = first + g.chunk < a.T ? first + g.chunk : a.T;
  float* const part = g.partials + (int64_t)(b / g.bands) * 2 * a.C + c;
  bool from_before = first > 0 && g.keys[first - 1] == g.keys[first];
  Eight sum{};
  for (int64_t i0 = first; i0 < last; i0 += kAhead) {
    v4u p[kAhead];
    uint32_t key[kAhead + 1];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t i = i0 + u < last ? i0 + u : last - 1;
      key[u] = g.keys[i];
      p[u] = v4u{0, 0, 0, 0};
      if (key[u] < (uint32_t)a.V)
        p[u] = __builtin_nontemporal_load(
            reinterpret_cast<const v4u*>(a.dy + (int64_t)g.positions[i] * a.lddy + c));
    }
    key[kAhead] = i0 + kAhead < a.T ? g.keys[i0 + kAhead] : 0xffffffffu;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i0 + u >= last || key[u] >= (uint32_t)a.V) break;  // (the tokens outside come last)
      Eight x;
      x.widen(p[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum.v[e] += x.v[e];
      const bool at_end = i0 + u + 1 == last;
      const uint32_t next = at_end ? (last < a.T ? g.keys[last] : 0xffffffffu) : key[u + 1];
      if (next == key[u] && !at_end) continue;
      if (next != key[u] && !from_before) {
        put_row(a, key[u], c, sum);
      } else {
        float* const to = part + (from_before ? 0 : a.C);
        *reinterpret_cast<float4*>(to) = make_float4(sum.v[0], sum.v[1], sum.v[2], sum.v[3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(sum.v[4], sum.v[5], sum.v[6], sum.v[7]);
      }
      sum = Eight{};
      from_before = false;
    }
  }
}

// Workgroup (chunk, band): if a run starts in the chunk and goes on into the next, its sums
// of all its chunks, added in order.
__global__ __launch_bounds__(kThreads) void embedding_join_kernel(Gradient g) {
  const EmbeddingBackwardArgs& a = g.a;
  const int64_t j = blockIdx.x / g.bands, c = (int64_t)(blockIdx.x % g.bands) * kBand + threadIdx.x * 8;
  const int64_t next = (j + 1) * g.chunk;  // (below T: the last chunk has no next)
  const uint32_t key = g.keys[next - 1];
  if (key >= (uint32_t)a.V || g.keys[next] != key) return;
  if (j > 0 && g.keys[j * g.chunk - 1] == key) return;  // it started before
  // the chunks after j whose first position is the run's: those up to j + more
  int more = 0;
  for (int64_t base = next;; base += (int64_t)kThreads * g.chunk) {
    const int64_t at = base + (int64_t)threadIdx.x * g.chunk;
    const int n = __syncthreads_count(at < a.T && g.keys[at < a.T ? at : 0] == key);
    more += n;
    if (n < kThreads) break;
  }
  if (c >= a.C) return;
  const float* part = g.partials + j * 2 * a.C + c;
  auto load = [&](const float* from) {
    const float4 lo = *reinterpret_cast<const float4*>(from), hi = *reinterpret_cast<const float4*>(from + 4);
    return Eight{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}};
  };
  Eight sum = load(part + a.C);
  for (int i0 = 1; i0 <= more; i0 += 4) {
    Eight x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = load(part + (int64_t)(i0 + u <= more ? i0 + u : more) * 2 * a.C);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u <= more)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum.v[e] += x[u].v[e];
  }
  put_row(a, key, c, sum);
}

// Positions of a chunk: 32, more where that leaves 2048 chunks or more.
inline int chunk_of(int64_t T) {
  int64_t n = 32;
  while (n * 2048 <= T) n *= 2;
  return (int)n;
}

inline int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

// The workspace's parts, in bytes from its start.
struct Layout {
  int64_t keys[2], positions[2], counts, bitmap, partials, bytes;
  int tiles;
  bool small;
  Layout(int64_t T, int64_t V, int64_t C) {
    small = T <= kSortMost && V < ((int64_t)1 << (32 - kPosBits));
    tiles = small ? 0 : (int)((T + kTile - 1) / kTile);
    int64_t at = 0;
    auto take = [&](int64_t n) {
      const int64_t here = at;
      at += round16(n);
      return here;
    };
    for (int i = 0; i < 2; ++i) {
      const bool used = i == 0 || !small;
      keys[i] = take(used ? 4 * T : 0);
      positions[i] = take(used ? 4 * T : 0);
    }
    counts = take((int64_t)4 * tiles << kWideDigit);
    bitmap = take((V + 31) / 32 * 4);
    const int64_t n = chunk_of(T);
    partials = take((T + n - 1) / n * 2 * C * 4);
    bytes = at;
  }
};

inline int bits_of(int64_t V) {  // of the keys 0 .. V
  int n = 0;
  while (V >> n) ++n;
  return n;
}

}  // namespace embedding_detail

using namespace embedding_detail;

hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t s) {
  const int bands = (int)((a.C + kBand - 1) / kBand);
  const unsigned grid = (unsigned)((a.T + kLookupRows - 1) / kLookupRows * bands);
  if (a.f32)
    embedding_kernel<true><<<grid, kThreads, 0, s>>>(a, bands);
  else
    embedding_kernel<false><<<grid, kThreads, 0, s>>>(a, bands);
  return hipGetLastError();
}

int64_t embedding_backward_workspace(int64_t T, int64_t V, int64_t C) { return Layout(T, V, C).bytes; }

hipError_t launch_embedding_backward(const EmbeddingBackwardArgs& a, hipStream_t s) {
  const Layout l(a.T, a.V, a.C);
  auto words = [&](int64_t at) { return reinterpret_cast<uint32_t*>(a.workspace + at); };
  uint32_t* const bitmap = words(l.bitmap);
  int out = 0;
  hipError_t e;
  if (l.small) {
    sort_small_kernel<<<1, kSortThreads, 0, s>>>(a.tokens, (int)a.T, a.V, bits_of(a.V), words(l.keys[0]),
                                                  words(l.positions[0]), bitmap);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    const int bits = bits_of(a.V);
    for (int shift = 0; shift < bits; shift += kWideDigit) {
      SortPass p{};
      p.tokens = shift == 0 ? a.tokens : nullptr;
      p.keys = words(l.keys[out]);
      p.positions = words(l.positions[out]);
      out ^= shift == 0 ? 0 : 1;
      p.keys_out = words(l.keys[out]);
      p.positions_out = words(l.positions[out]);
      p.counts = words(l.counts);
      p.T = a.T;
      p.V = a.V;
      p.tiles = l.tiles;
      p.shift = shift;
      p.bitmap = shift + kWideDigit >= bits ? bitmap : nullptr;
      sort_count_kernel<<<l.tiles, kTileThreads, 0, s>>>(p);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      sort_scan_kernel<<<1, kSortThreads, 0, s>>>(p.counts, (int64_t)l.tiles << kWideDigit);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      sort_move_kernel<<<l.tiles, kTileThreads, 0, s>>>(p);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  Gradient g;
  g.a = a;
  g.keys = words(l.keys[out]);
  g.positions = words(l.positions[out]);
  g.bitmap = bitmap;
  g.partials = reinterpret_cast<float*>(a.workspace + l.partials);
  g.chunk = chunk_of(a.T);
  g.chunks = (int)((a.T + g.chunk - 1) / g.chunk);
  g.bands = (int)((a.C + kBand - 1) / kBand);
  const int64_t fill = a.accumulate ? 0 : (a.V + kFillRows - 1) / kFillRows;
  embedding_sums_kernel<<<(unsigned)((g.chunks + fill) * g.bands), kThreads, 0, s>>>(g);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (g.chunks > 1) {
    embedding_join_kernel<<<(unsigned)((int64_t)(g.chunks - 1) * g.bands), kThreads, 0, s>>>(g);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace fp8q
