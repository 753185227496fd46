// The embedding table's rows for a batch of tokens, and the table's gradient, on gfx950.
//
//   y[t] = scale w[token_t],    dw[v] = scale sum over token_t = v of dy[t]
//
// A token outside 0 .. V-1 (padding) gives a row of zeros and takes no part in the gradient.
//
// The gradient sums each row in the order of t, in fp32, so that every run gives the same bits.
// Up to kFewTokens tokens are compared with each other (embedding_few_kernel, see takes_few).  More are sorted
// (stably: by token, then by t), the sorted positions are cut into chunks, and a workgroup adds up
// the rows of dy of one chunk, over a band of columns, run by run of equal tokens.  A run inside a
// chunk goes to the table at once; one that crosses chunks leaves a sum per chunk in the workspace,
// and a second kernel adds those in order.  The rows of tokens that do not occur are filled with zeros by a
// launch between the sort, which leaves a bitmap of those that do, and the sums: most of what a whole
// gradient costs.  Bound by HBM, V C elements written and T C read: 16384 tokens, 131072 x 4096 fp32 409
// us, of them the sort 13, zeros 303 (7.1 TB/s), sums 84 and their join 6.  Small tables wait for the chain of
// launches: 5003 tokens, 32000 x 2048 bf16, twice, 77 us (sorts 7, zeros 18, sums 8 and 11, joins 7) where the
// bytes would take 23.
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
  // the rows' tokens, one a lane, in one load; -1: padding
  const int lane = threadIdx.x & 63;
  int64_t token = -1;
  if (lane < kLookupRows && t0 + lane < a.T) token = a.tokens[t0 + lane];
  const int index = token >= 0 && token < a.V ? (int)token : -1;
  int v[kLookupRows];
#pragma unroll
  for (int i = 0; i < kLookupRows; ++i) v[i] = __builtin_amdgcn_readlane(index, i);
  if (c >= a.C) return;
  v4u p[kLookupRows], q[kLookupRows];
#pragma unroll
  for (int i = 0; i < kLookupRows; ++i) {
    p[i] = q[i] = v4u{0, 0, 0, 0};
    if (v[i] < 0) continue;
    if constexpr (F32) {
      const v4u* const from = reinterpret_cast<const v4u*>(static_cast<const float*>(a.weight) + v[i] * a.ldw + c);
      p[i] = from[0];
      q[i] = from[1];
    } else {
      p[i] = *reinterpret_cast<const v4u*>(static_cast<const uint16_t*>(a.weight) + v[i] * a.ldw + c);
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
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = v[i] >= 0 ? x.v[e] * a.scale : 0.0f;
    *reinterpret_cast<v4u*>(a.y + (t0 + i) * a.ldy + c) = x.narrow();
  }
}

// ---- the sort -----------------------------------------------------------------------------
//
// Radix sort by the token, least significant digit first; tokens outside the vocabulary take
// the key V.  A wave ranks 64 keys at a time, in order: the lanes with its digit are found by
// a ballot per bit, the count of those before them in the wave from a counter in LDS.

// The lanes whose BITS-bit digit is this lane's (of those that are live): a bit's ballot,
// inverted in the lanes that have it clear, leaves the others out.
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool live) {
  const uint64_t all = __ballot(live);
  uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const uint32_t clear = (digit >> b & 1) - 1;  // all ones where the bit is clear
    const uint64_t o = __ballot(clear == 0);
    lo &= (uint32_t)o ^ clear;
    hi &= (uint32_t)(o >> 32) ^ clear;
  }
  return (uint64_t)hi << 32 | lo;
}

// A wave's LDS operations before this point come before those after it, for all its lanes.
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// This lane's place among its wave's keys of the same digit so far (counters: the wave's, by
// digit), and the counter moved on.
template <int BITS>
__device__ __forceinline__ uint32_t rank_in_wave(uint32_t digit, bool live, uint32_t* counters) {
  const uint64_t m = same_digit<BITS>(digit, live);
  const uint32_t below =
      __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
  uint32_t before = 0;
  if (live) before = counters[digit];
  in_order();
  if (live && below == 0) counters[digit] = before + (uint32_t)__popcll(m);
  in_order();
  return before + below;
}

__device__ __forceinline__ uint32_t key_of(int64_t token, int64_t V) {
  return token >= 0 && token < V ? (uint32_t)token : (uint32_t)V;
}

// Which tokens occur: bit v / kClasses of part v % kClasses, parts of used_words(V) words.
constexpr int kClassBits = 6, kClasses = 1 << kClassBits;
__host__ __device__ constexpr int64_t used_words(int64_t V) { return (V + 32 * kClasses - 1) / (32 * kClasses); }
__device__ __forceinline__ bool occurs(const uint32_t* used, int64_t V, uint64_t v) {
  return used[(v & (kClasses - 1)) * used_words(V) + (v >> (kClassBits + 5))] >> (v >> kClassBits & 31) & 1;
}

// Up to kSortMost tokens: workgroup g takes those with token % kClasses = g out of all and sorts
// them by token / kClasses, its place in the whole being after those of the workgroups before it
// (equal tokens stay together, which is all that the sums ask for).  16384 tokens with frequencies of 1 /
// rank in one workgroup 25 us, in eight 19, in 64 17 (before what is said below).  Tokens outside the vocabulary are the
// last of the last class.  A word holds
// key and t together (kPosBits for t), so the pass that a key makes is one word through LDS.  Wave w has the words
// from w 64 rounds on, so that its rounds go in order.
//
// What it waits for is its own chain, and of that much is code that is met for the first time: a chain of rounds that
// are skipped costs as much as one that works.  So the kernel has as many rounds as T asks for, 4, 8 or 16, and
// sorts in two where its class has no more keys than that (5003 tokens 6.6 us, with 16 rounds throughout 11.0;
// 16384 13.9 and 16.6).
constexpr int kSortThreads = 1024, kSortWaves = 16, kSortRounds = 16, kFewRounds = 2, kPosBits = 14;
constexpr int64_t kSortMost = 16384;
constexpr int kDigit = 9;  // bits a pass, at most
constexpr int kUsedLds = 1024;  // words of a part of the bitmap in LDS
static_assert(kUsedLds * 32 < 1 << (32 - kPosBits));  // (their keys, and that of the tokens outside, fit beside t)

struct SmallSort {
  uint32_t words[kSortMost];
  uint32_t counters[kSortWaves][1 << kDigit], sums[kSortWaves], lower[kSortWaves];
  uint32_t marks[kUsedLds];
};

struct SmallSortArgs {
  const int64_t* tokens;
  int T, key_bits;
  int64_t V;
  uint32_t *keys, *positions, *used;
};

// The class's n words, of up to ROUNDS rounds, sorted in LDS and written from `place` on.
template <int ROUNDS>
__device__ __forceinline__ void sort_class(SmallSort& s, const SmallSortArgs& a, int n, uint32_t place) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int rounds = (n + kSortThreads - 1) / kSortThreads, first = wave * rounds * 64 + lane;
  uint32_t w[ROUNDS], rank[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    w[r] = 0xffffffffu;
    if (r < rounds && first + r * 64 < n) w[r] = s.words[first + r * 64];
  }
  const int passes = (a.key_bits + kDigit - 1) / kDigit, bits = (a.key_bits + passes - 1) / passes;
  uint32_t* const mine = s.counters[wave];
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = kPosBits + pass * bits;
    auto digit_of = [&](uint32_t x) { return x >> shift & ((1u << bits) - 1); };
    for (int d = lane; d < 1 << kDigit; d += 64) mine[d] = 0;
    in_order();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (r < rounds) rank[r] = rank_in_wave<kDigit>(digit_of(w[r]), first + r * 64 < n, mine);
    __syncthreads();
    // prefix sums over the digits, and over the waves of a digit: two threads a digit
    constexpr int kPer = kSortWaves / 2;
    static_assert(2 << kDigit == kSortThreads);
    uint32_t c[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      c[i] = s.counters[(t & 1) * kPer + i][t >> 1];
      sum += c[i];
    }
    uint32_t scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = __shfl_up(scan, d, 64);
      if (lane >= d) scan += o;
    }
    if (lane == 63) s.sums[wave] = scan;
    __syncthreads();
    uint32_t base = scan - sum;
#pragma unroll
    for (int o = 0; o < kSortWaves; ++o) base += o < wave ? s.sums[o] : 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      s.counters[(t & 1) * kPer + i][t >> 1] = base;
      base += c[i];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (r < rounds && first + r * 64 < n) s.words[mine[digit_of(w[r])] + rank[r]] = w[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (r < rounds && first + r * 64 < n) w[r] = s.words[first + r * 64];
    // (the next pass writes the words again only after more barriers)
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = first + r * 64;
    if (r < rounds && i < n) {
      const uint32_t high = w[r] >> kPosBits, key = high << kClassBits | blockIdx.x;
      a.keys[place + i] = key;
      a.positions[place + i] = w[r] & ((1u << kPosBits) - 1);
      if (key < (uint32_t)a.V)
        __hip_atomic_fetch_or(s.marks + (high >> 5), 1u << (high & 31), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
  }
}

template <int ROUNDS>
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(SmallSortArgs a) {
  __shared__ SmallSort s;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t g = blockIdx.x;
  uint32_t key[ROUNDS];
  const int rounds = (a.T + kSortThreads - 1) / kSortThreads, first = wave * rounds * 64 + lane;
  const uint32_t outside = (uint32_t)((a.V + kClasses - 1) / kClasses * kClasses + kClasses - 1);
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = first + r * 64;
    int64_t token = 0;
    if (r < rounds && i < a.T) token = a.tokens[i];
    key[r] = token >= 0 && token < a.V ? (uint32_t)token : outside;
  }
  s.marks[t] = 0;
  static_assert(kUsedLds == kSortThreads);
  // this class's words, in order
  uint32_t own = 0, less = 0;
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const bool live = r < rounds && first + r * 64 < a.T;
    own += (uint32_t)__popcll(__ballot(live && (key[r] & (kClasses - 1)) == g));
    less += (uint32_t)__popcll(__ballot(live && (key[r] & (kClasses - 1)) < g));
  }
  if (lane == 0) {
    s.sums[wave] = own;
    s.lower[wave] = less;
  }
  __syncthreads();
  uint32_t at = 0, place = 0, count = 0;
#pragma unroll
  for (int o = 0; o < kSortWaves; ++o) {
    at += o < wave ? s.sums[o] : 0;
    count += s.sums[o];
    place += s.lower[o];
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const bool mine = r < rounds && first + r * 64 < a.T && (key[r] & (kClasses - 1)) == g;
    const uint64_t m = __ballot(mine);
    if (mine)
      s.words[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0))] =
          key[r] >> kClassBits << kPosBits | (uint32_t)(first + r * 64);
    at += (uint32_t)__popcll(m);
  }
  __syncthreads();
  const int n = __builtin_amdgcn_readfirstlane((int)count);
  if (n <= kFewRounds * kSortThreads)
    sort_class<kFewRounds>(s, a, n, place);
  else
    sort_class<ROUNDS>(s, a, n, place);
  __syncthreads();
  const int64_t part = used_words(a.V);
  if (t < part) a.used[g * part + t] = s.marks[t];
}

// More tokens: a workgroup takes a tile of them, up to kTiles tiles, and a pass is two launches, the tiles'
// counts by digit and the words to their places, where every workgroup adds up the counts before its own.
// The first pass reads the tokens.  18888 tokens of 18212: two passes and the bitmap 23 us; with a third launch for
// the counts' sums, tiles of 4096 and the bitmap from every token about 75.
constexpr int kWideThreads = 512, kWideWaves = 8, kWideDigit = 9, kWideAhead = 4;
static_assert(kWideThreads == 1 << kWideDigit);  // (thread d has digit d)
constexpr int64_t kTiles = 128, kTileStep = 2 * kWideThreads;

// Tokens of a tile: whole rounds of every wave.
inline int64_t tile_of(int64_t T) { return ((T + kTiles - 1) / kTiles + kTileStep - 1) / kTileStep * kTileStep; }

struct SortPass {
  const int64_t* tokens;  // of the first pass, else null
  const uint32_t *keys, *positions;
  uint32_t *keys_out, *positions_out;
  uint32_t* counts;  // [tiles][512]
  int64_t T, V;
  int tile, tiles, shift;
  uint32_t* used;  // of the first pass of a whole gradient, else null: cleared
  __device__ __forceinline__ uint32_t key(int64_t i) const { return tokens ? key_of(tokens[i], V) : keys[i]; }
  __device__ __forceinline__ uint32_t digit(uint32_t k) const { return k >> shift & ((1u << kWideDigit) - 1); }
};

__global__ __launch_bounds__(kWideThreads) void sort_count_kernel(SortPass p) {
  __shared__ uint32_t counts[1 << kWideDigit];
  const int t = threadIdx.x;
  counts[t] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * p.tile, last = first + p.tile < p.T ? first + p.tile : p.T;
  for (int64_t i0 = first + t; i0 < last; i0 += kWideAhead * kWideThreads) {
    uint32_t key[kWideAhead];
#pragma unroll
    for (int u = 0; u < kWideAhead; ++u) {
      const int64_t i = i0 + u * kWideThreads;
      key[u] = i < last ? p.key(i) : 0;
    }
#pragma unroll
    for (int u = 0; u < kWideAhead; ++u)
      if (i0 + u * kWideThreads < last)
        __hip_atomic_fetch_add(counts + p.digit(key[u]), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  __syncthreads();
  p.counts[(int64_t)blockIdx.x * kWideThreads + t] = counts[t];
  if (p.used)
    for (int64_t i = (int64_t)blockIdx.x * kWideThreads + t; i < kClasses * used_words(p.V);
         i += (int64_t)gridDim.x * kWideThreads)
      p.used[i] = 0;
}

__global__ __launch_bounds__(kWideThreads) void sort_move_kernel(SortPass p) {
  __shared__ uint32_t counters[kWideWaves][1 << kWideDigit], sums[kWideWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
#pragma unroll
  for (int w = 0; w < kWideWaves; ++w) counters[w][t] = 0;
  __syncthreads();
  // this wave's part of the tile
  const int per = p.tile / kWideWaves;
  const int64_t first = (int64_t)blockIdx.x * p.tile + wave * per;
  const int64_t last = first + per < p.T ? first + per : p.T;
  auto each = [&](auto&& f) {
    for (int64_t i0 = first; i0 < last; i0 += kWideAhead * 64) {
      uint32_t key[kWideAhead], position[kWideAhead];
#pragma unroll
      for (int u = 0; u < kWideAhead; ++u) {
        const int64_t i = i0 + u * 64 + lane;
        key[u] = i < last ? p.key(i) : 0;
        position[u] = p.tokens || i >= last ? (uint32_t)i : p.positions[i];
      }
#pragma unroll
      for (int u = 0; u < kWideAhead; ++u)
        if (i0 + u * 64 < last) f(key[u], position[u], i0 + u * 64 + lane < last);
    }
  };
  each([&](uint32_t key, uint32_t, bool live) {
    if (live) __hip_atomic_fetch_add(&counters[wave][p.digit(key)], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  });
  // this thread's digit in the tiles before, and in all
  uint32_t before = 0, all = 0;
#pragma unroll 8
  for (int b = 0; b < p.tiles; ++b) {
    const uint32_t c = p.counts[(int64_t)b * kWideThreads + t];
    before += b < (int)blockIdx.x ? c : 0;
    all += c;
  }
  uint32_t scan = all;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(scan, d, 64);
    if (lane >= d) scan += o;
  }
  if (lane == 63) sums[wave] = scan;
  __syncthreads();
  uint32_t base = scan - all + before;
#pragma unroll
  for (int w = 0; w < kWideWaves; ++w) base += w < wave ? sums[w] : 0;
  // where each wave's words of the digit start
#pragma unroll
  for (int w = 0; w < kWideWaves; ++w) {
    const uint32_t c = counters[w][t];
    counters[w][t] = base;
    base += c;
  }
  __syncthreads();
  each([&](uint32_t key, uint32_t position, bool live) {
    const uint32_t to = rank_in_wave<kWideDigit>(p.digit(key), live, counters[wave]);
    if (live) {
      p.keys_out[to] = key;
      p.positions_out[to] = position;
    }
  });
}

// The bitmap of the tokens that occur, from the sorted keys (the first of each run).
__global__ __launch_bounds__(kThreads) void sort_mark_kernel(const uint32_t* keys, int64_t T, int64_t V, uint32_t* used) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= T) return;
  const uint32_t key = keys[i], high = key >> kClassBits;
  if (key >= (uint32_t)V || (i > 0 && keys[i - 1] == key)) return;
  __hip_atomic_fetch_or(used + (key & (kClasses - 1)) * used_words(V) + (high >> 5), 1u << (high & 31), __ATOMIC_RELAXED,
                        __HIP_MEMORY_SCOPE_AGENT);
}

// ---- the sums -----------------------------------------------------------------------------

// n / d for n below 2^36, d below 2^29, by a product: with k = 36 + the bits of d, m = ceil(2^k /
// d) is off by less than d, so n m / 2^k by less than 1 / d.
struct Divisor {
  uint32_t d;
  int shift;
  uint64_t m;
  explicit Divisor(uint32_t d_ = 1) : d(d_), shift(36) {
    while ((uint64_t)1 << (shift - 36) < d) ++shift;
    m = (uint64_t)((((unsigned __int128)1 << shift) + d - 1) / d);
  }
  __device__ __forceinline__ uint64_t quotient(uint64_t n) const {
    const uint64_t lo = n * m, hi = __umul64hi(n, m);
    return shift >= 64 ? hi >> (shift - 64) : hi << (64 - shift) | lo >> shift;
  }
};

struct Gradient {
  EmbeddingBackwardArgs a;
  const uint32_t *keys, *positions, *used;
  float* partials;  // [chunks][2][C]: the sums of a run from the chunk before, and of one into the next
  int chunk;        // positions of a chunk
  int chunks, bands;
  Divisor row;      // 16-byte pieces of a row of the table
};

// Zeros in the rows that no token names, in all without a bitmap: one 16-byte piece a thread, workgroup after workgroup
// along the table (2 GiB 303 us, 7.1 TB/s; in a probe, back to back with the gaps between launches, 319, four
// pieces a thread 363, workgroups that stay 378 to 433).
template <bool F32>
__global__ __launch_bounds__(kThreads) void embedding_fill_kernel(Gradient g) {
  const EmbeddingBackwardArgs& a = g.a;
  const unsigned group = blockIdx.x;
  constexpr int kN = F32 ? 4 : 8;
  // the workgroup's first piece's row, and this thread's from there
  const uint64_t first = (uint64_t)group * kThreads;
  uint64_t v = g.row.quotient(first);
  int64_t c = (int64_t)(first - v * g.row.d) + threadIdx.x;
  const uint32_t more = g.row.quotient((uint64_t)c);
  v += more;
  c -= (int64_t)more * g.row.d;
  if (v >= (uint64_t)a.V) return;
  if (g.used && occurs(g.used, a.V, v)) return;
  const int64_t at = (int64_t)v * a.ldw + c * kN;
  const v4u zero = {0, 0, 0, 0};
  if constexpr (F32)
    *reinterpret_cast<v4u*>(static_cast<float*>(a.dweight) + at) = zero;
  else
    *reinterpret_cast<v4u*>(static_cast<uint16_t*>(a.dweight) + at) = zero;
}

// A thread's eight columns of a band, in two pieces of four: side by side for a bf16 table,
// kHalf apart for an fp32 one, so that a store of four is beside its neighbours'.
constexpr int kHalf = kBand / 2;
template <bool F32>
__device__ __forceinline__ int64_t column(int64_t band) {
  return band * kBand + threadIdx.x * (F32 ? 4 : 8);
}

// As they are in memory: to be widened where they are used, so that a load waits for no other's.
template <bool F32>
__device__ __forceinline__ v4u load_dy(const uint16_t* row, bool second) {
  if constexpr (F32) {
    const uint2 lo = *reinterpret_cast<const uint2*>(row);
    const uint2 hi = second ? *reinterpret_cast<const uint2*>(row + kHalf) : make_uint2(0, 0);
    return v4u{lo.x, lo.y, hi.x, hi.y};
  } else {
    return *reinterpret_cast<const v4u*>(row);
  }
}

// What the columns of row v of the table from c on hold (second: the other four are inside it, too).
template <bool F32>
struct TableRow {
  v4u p[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const EmbeddingBackwardArgs& a, uint32_t v, int64_t c, bool second) {
    const int64_t at = (int64_t)v * a.ldw + c;
    if constexpr (F32) {
      const float* const from = static_cast<const float*>(a.dweight) + at;
      p[0] = *reinterpret_cast<const v4u*>(from);
      if (second) p[1] = *reinterpret_cast<const v4u*>(from + kHalf);
    } else {
      p[0] = *reinterpret_cast<const v4u*>(static_cast<const uint16_t*>(a.dweight) + at);
    }
  }
  __device__ __forceinline__ Eight eight() const {
    Eight x;
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x.v[e] = __uint_as_float(p[0][e]);
        x.v[4 + e] = __uint_as_float(p[1][e]);
      }
    } else {
      x.widen(p[0]);
    }
    return x;
  }
};

template <bool F32, bool ADD>
__device__ __forceinline__ void put_row(const EmbeddingBackwardArgs& a, uint32_t v, int64_t c, bool second,
                                        const Eight& sum, const TableRow<F32>& row) {
  const int64_t at = (int64_t)v * a.ldw + c;
  Eight x, old{};
  if (ADD) old = row.eight();
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = ADD ? old.v[e] + sum.v[e] * a.scale : sum.v[e] * a.scale;
  if constexpr (F32) {
    float* const to = static_cast<float*>(a.dweight) + at;
    v4u lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = __float_as_uint(x.v[e]);
      hi[e] = __float_as_uint(x.v[4 + e]);
    }
    __builtin_nontemporal_store(lo, reinterpret_cast<v4u*>(to));
    if (second) __builtin_nontemporal_store(hi, reinterpret_cast<v4u*>(to + kHalf));
  } else {
    __builtin_nontemporal_store(x.narrow(), reinterpret_cast<v4u*>(static_cast<uint16_t*>(a.dweight) + at));
  }
}

// A workgroup sums a chunk over a band of columns, kAhead positions at a time: their rows of dy
// and, to be added to, the table's rows of the runs that end there are all in flight together.  A wave reads the
// keys and positions of 64 at once, one a lane, and has them as scalars from there: read one by one, each for
// the whole wave, they and the rows waited for each other (40000 x 1024 bf16 68 us, so 37; 16384 x 4096 for an
// fp32 table 98 and 84).
constexpr int kChunk = 8;  // a chunk has a multiple of it
constexpr int kAhead = 8;

template <bool F32, bool ADD>
__global__ __launch_bounds__(kThreads) void embedding_sums_kernel(Gradient g) {
  const EmbeddingBackwardArgs& a = g.a;
  const int64_t j = blockIdx.x / g.bands;
  int64_t c = column<F32>(blockIdx.x % g.bands);
  const bool inside = c < a.C;
  if (!__any(inside)) return;
  if (!inside) c = 0;  // (lanes that store nothing)
  const bool second = !F32 || c + kHalf < a.C;
  const int64_t first = j * g.chunk, last = first + g.chunk < a.T ? first + g.chunk : a.T;
  float* const part = g.partials + j * 2 * a.C + c;
  const uint32_t V = (uint32_t)a.V;
  const int lane = threadIdx.x & 63;
  bool from_before = first > 0 && g.keys[first - 1] == g.keys[first];
  Eight sum{};
  for (int64_t block = first; block < last; block += 64) {
    const int64_t i = block + lane;
    const uint32_t keys = i < a.T ? g.keys[i] : 0xffffffffu, nexts = i + 1 < a.T ? g.keys[i + 1] : 0xffffffffu,
                   positions = i < a.T ? g.positions[i] : 0;
    const int n = last - block < 64 ? (int)(last - block) : 64;
    for (int i0 = 0; i0 < n; i0 += kAhead) {
      v4u x[kAhead];
      TableRow<F32> old[kAhead];
      uint32_t key[kAhead], next[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        key[u] = __builtin_amdgcn_readlane(keys, i0 + u);
        next[u] = __builtin_amdgcn_readlane(nexts, i0 + u);
        x[u] = v4u{0, 0, 0, 0};
        old[u] = TableRow<F32>{};
        if (key[u] < V) {
          x[u] = load_dy<F32>(a.dy + (int64_t)__builtin_amdgcn_readlane(positions, i0 + u) * a.lddy + c, second);
          if (ADD && next[u] != key[u]) old[u].load(a, key[u], c, second);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (key[u] >= V) break;  // (the tokens outside come last)
        Eight now;
        now.widen(x[u]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum.v[e] += now.v[e];
        const bool ends = next[u] != key[u];
        if (!ends && block + i0 + u + 1 != last) continue;
        if (inside && ends && !from_before) {
          put_row<F32, ADD>(a, key[u], c, second, sum, old[u]);
        } else if (inside) {
          float* const to = part + (from_before ? 0 : a.C);
          *reinterpret_cast<float4*>(to) = make_float4(sum.v[0], sum.v[1], sum.v[2], sum.v[3]);
          if (second)
            *reinterpret_cast<float4*>(to + (F32 ? kHalf : 4)) = make_float4(sum.v[4], sum.v[5], sum.v[6], sum.v[7]);
        }
        sum = Eight{};
        from_before = false;
      }
    }
  }
}

// Workgroup (chunk, band): if a run starts in the chunk and goes on into the next, its sums
// of all its chunks, added in order.
template <bool F32, bool ADD>
__global__ __launch_bounds__(kThreads) void embedding_join_kernel(Gradient g) {
  const EmbeddingBackwardArgs& a = g.a;
  const int64_t j = blockIdx.x / g.bands, c = column<F32>(blockIdx.x % g.bands);
  const int64_t next = (j + 1) * g.chunk;  // (below T: the last chunk has no next)
  // (three keys in one load: the chunk's last, the next one's first, and the one before the chunk; and beside
  // it the first of each of 64 chunks, the next one on)
  const int lane = threadIdx.x & 63;
  const int64_t here = lane == 0 ? next - 1 : (lane == 1 ? next : j * g.chunk - 1);
  const uint32_t three = here >= 0 ? g.keys[here] : 0xffffffffu;
  const int64_t there = next + (int64_t)lane * g.chunk;
  const uint32_t firsts = there < a.T ? g.keys[there] : 0xffffffffu;
  const uint32_t key = __builtin_amdgcn_readlane(three, 0), after = __builtin_amdgcn_readlane(three, 1),
                 before = __builtin_amdgcn_readlane(three, 2);
  if (key >= (uint32_t)a.V || after != key || before == key) return;  // none, or it started before
  // the chunks after j whose first position is the run's: those up to j + more
  int more = __popcll(__ballot(firsts == key));
  for (int64_t base = next; more % 64 == 0;) {
    base += (int64_t)64 * g.chunk;
    const int64_t at = base + (int64_t)lane * g.chunk;
    const int n = __popcll(__ballot(at < a.T && g.keys[at < a.T ? at : 0] == key));
    more += n;
    if (n == 0) break;
  }
  if (c >= a.C) return;
  const bool second = !F32 || c + kHalf < a.C;
  const float* part = g.partials + j * 2 * a.C + c;
  auto load = [&](const float* from) {
    const float4 lo = *reinterpret_cast<const float4*>(from);
    const float4 hi = second ? *reinterpret_cast<const float4*>(from + (F32 ? kHalf : 4)) : make_float4(0, 0, 0, 0);
    return Eight{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}};
  };
  Eight sum = load(part + a.C);
  TableRow<F32> old{};
  if (ADD) old.load(a, key, c, second);
  constexpr int kParts = 16;
  for (int i0 = 1; i0 <= more; i0 += kParts) {
    Eight x[kParts];
#pragma unroll
    for (int u = 0; u < kParts; ++u) x[u] = load(part + (int64_t)(i0 + u <= more ? i0 + u : more) * 2 * a.C);
#pragma unroll
    for (int u = 0; u < kParts; ++u)
      if (i0 + u <= more)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum.v[e] += x[u].v[e];
  }
  put_row<F32, ADD>(a, key, c, second, sum, old);
}

// Few tokens: workgroup (t, band) sums its token's rows if none before t is the same; every wave finds
// them by comparing all tokens with its own.  Two launches in place of four, one in place of three: 256 tokens
// with frequencies of 1 / rank, 32000 x 2048 bf16, 22.6 us, sorted 31.7, added 4.8 and 13.4; only where most
// are the same does it take longer (all of them: 44.5 and 33.7, added 22.4 and 15.0).
constexpr int kFewTokens = 256, kFewAhead = 16;

template <bool F32, bool ADD>
__global__ __launch_bounds__(kThreads) void embedding_few_kernel(Gradient g) {
  __shared__ uint16_t lists[kThreads / 64][kFewTokens];
  const EmbeddingBackwardArgs& a = g.a;
  const int t = blockIdx.x / g.bands, lane = threadIdx.x & 63;
  constexpr int kGroups = kFewTokens / 64;
  uint32_t keys[kGroups], key = 0;
#pragma unroll
  for (int q = 0; q < kGroups; ++q) {
    const int i = q * 64 + lane;
    keys[q] = i < a.T ? key_of(a.tokens[i], a.V) : 0xffffffffu;
  }
#pragma unroll
  for (int q = 0; q < kGroups; ++q)
    if (q == t >> 6) key = __builtin_amdgcn_readlane(keys[q], t & 63);
  if (key >= (uint32_t)a.V) return;
  uint16_t* const list = lists[threadIdx.x >> 6];
  int n = 0;
#pragma unroll
  for (int q = 0; q < kGroups; ++q) {
    const uint64_t same = __ballot(keys[q] == key);
    if (keys[q] == key)
      list[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0))] =
          (uint16_t)(q * 64 + lane);
    n += __popcll(same);
  }
  in_order();
  if (__builtin_amdgcn_readfirstlane(list[0]) != t) return;
  int64_t c = column<F32>(blockIdx.x % g.bands);
  const bool inside = c < a.C;
  if (!__any(inside)) return;
  if (!inside) c = 0;  // (lanes that store nothing)
  const bool second = !F32 || c + kHalf < a.C;
  TableRow<F32> old{};
  if (ADD) old.load(a, key, c, second);
  Eight sum{};
  for (int i0 = 0; i0 < n; i0 += kFewAhead) {
    v4u x[kFewAhead];
    const int rows = lane < kFewAhead && i0 + lane < n ? list[i0 + lane] : 0;
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      x[u] = v4u{0, 0, 0, 0};  // (zeros change no sum)
      if (i0 + u < n) x[u] = load_dy<F32>(a.dy + __builtin_amdgcn_readlane(rows, u) * a.lddy + c, second);
    }
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      Eight now;
      now.widen(x[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum.v[e] += now.v[e];
    }
  }
  if (inside) put_row<F32, ADD>(a, key, c, second, sum, old);
}

inline int64_t bands_of(int64_t C) { return (C + kBand - 1) / kBand; }

// Whether tokens are compared and not sorted: few of them, in rows whose bands leave the launch's threads below 2^32.
inline bool takes_few(int64_t T, int64_t C) {
  return T <= kFewTokens && T * bands_of(C) < ((int64_t)1 << 32) / kThreads;
}

// Positions of a chunk, kChunk or a power of two times it: doubled while as many as they are make 2048 workgroups or
// more, so that 1024 to 2047 are left (fewer where there were fewer, or at the most positions of a chunk).
inline int chunk_of(int64_t T, int64_t C) {
  int64_t n = kChunk;
  while (n * 2048 <= T * bands_of(C) && n < ((int64_t)1 << 20)) n *= 2;
  return (int)n;
}

inline int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

// The workspace's parts, in bytes from its start.
struct Layout {
  int64_t keys[2], positions[2], counts, used, partials, bytes;
  int tile, tiles;
  bool small;
  Layout(int64_t T, int64_t V, int64_t C) {
    small = T <= kSortMost && used_words(V) <= kUsedLds;
    tile = small ? 0 : (int)tile_of(T);
    tiles = small ? 0 : (int)((T + tile - 1) / tile);
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
    used = take(4 * kClasses * used_words(V));
    const int64_t n = chunk_of(T, C);
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
  const int bands = (int)bands_of(a.C);
  const unsigned grid = (unsigned)((a.T + kLookupRows - 1) / kLookupRows * bands);
  if (a.f32)
    embedding_kernel<true><<<grid, kThreads, 0, s>>>(a, bands);
  else
    embedding_kernel<false><<<grid, kThreads, 0, s>>>(a, bands);
  return hipGetLastError();
}

// (tokens that are compared leave nothing in it: one piece, so that it has an address)
int64_t embedding_backward_workspace(int64_t T, int64_t V, int64_t C) {
  return takes_few(T, C) ? 16 : Layout(T, V, C).bytes;
}

hipError_t launch_embedding_backward(const EmbeddingBackwardArgs& a, hipStream_t s) {
  const int bands = (int)bands_of(a.C);
  Gradient g;
  g.a = a;
  g.bands = bands;
  g.row = Divisor((uint32_t)(a.C / (a.f32 ? 4 : 8)));
  const int64_t pieces = (a.V * g.row.d + kThreads - 1) / kThreads;
  const auto fill = [&] {
    if (a.accumulate) return hipSuccess;
    if (a.f32)
      embedding_fill_kernel<true><<<(unsigned)pieces, kThreads, 0, s>>>(g);
    else
      embedding_fill_kernel<false><<<(unsigned)pieces, kThreads, 0, s>>>(g);
    return hipGetLastError();
  };
  hipError_t e;
  if (takes_few(a.T, a.C)) {
    g.used = nullptr;
    if ((e = fill()) != hipSuccess) return e;
    const unsigned grid = (unsigned)(a.T * bands);
    if (a.accumulate && a.f32)
      embedding_few_kernel<true, true><<<grid, kThreads, 0, s>>>(g);
    else if (a.accumulate)
      embedding_few_kernel<false, true><<<grid, kThreads, 0, s>>>(g);
    else if (a.f32)
      embedding_few_kernel<true, false><<<grid, kThreads, 0, s>>>(g);
    else
      embedding_few_kernel<false, false><<<grid, kThreads, 0, s>>>(g);
    return hipGetLastError();
  }
  const Layout l(a.T, a.V, a.C);
  auto words = [&](int64_t at) { return reinterpret_cast<uint32_t*>(a.workspace + at); };
  int out = 0;
  if (l.small) {
    const SmallSortArgs p{a.tokens, (int)a.T, bits_of((a.V + kClasses - 1) / kClasses), a.V,
                          words(l.keys[0]), words(l.positions[0]), words(l.used)};
    if (a.T <= 4 * kSortThreads)
      sort_small_kernel<4><<<kClasses, kSortThreads, 0, s>>>(p);
    else if (a.T <= 8 * kSortThreads)
      sort_small_kernel<8><<<kClasses, kSortThreads, 0, s>>>(p);
    else
      sort_small_kernel<kSortRounds><<<kClasses, kSortThreads, 0, s>>>(p);
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
      p.tile = l.tile;
      p.tiles = l.tiles;
      p.shift = shift;
      p.used = shift == 0 && !a.accumulate ? words(l.used) : nullptr;
      sort_count_kernel<<<l.tiles, kWideThreads, 0, s>>>(p);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      sort_move_kernel<<<l.tiles, kWideThreads, 0, s>>>(p);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (!a.accumulate) {
      sort_mark_kernel<<<(unsigned)((a.T + kThreads - 1) / kThreads), kThreads, 0, s>>>(words(l.keys[out]), a.T, a.V,
                                                                                        words(l.used));
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  g.keys = words(l.keys[out]);
  g.positions = words(l.positions[out]);
  g.used = words(l.used);
  g.partials = reinterpret_cast<float*>(a.workspace + l.partials);
  g.chunk = chunk_of(a.T, a.C);
  g.chunks = (int)((a.T + g.chunk - 1) / g.chunk);
  const auto launch = [&](auto sums, auto join) {
    if (const hipError_t st = fill(); st != hipSuccess) return st;
    sums<<<(unsigned)(g.chunks * g.bands), kThreads, 0, s>>>(g);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess || g.chunks == 1) return st;
    join<<<(unsigned)((g.chunks - 1) * g.bands), kThreads, 0, s>>>(g);
    return hipGetLastError();
  };
  if (a.accumulate)
    return a.f32 ? launch(embedding_sums_kernel<true, true>, embedding_join_kernel<true, true>)
                 : launch(embedding_sums_kernel<false, true>, embedding_join_kernel<false, true>);
  return a.f32 ? launch(embedding_sums_kernel<true, false>, embedding_join_kernel<true, false>)
               : launch(embedding_sums_kernel<false, false>, embedding_join_kernel<false, false>);
}

}  // namespace fp8q
