// C-ABI of the 4-bit rollout's operators and of the two ends of the policy: argument
// validation, then kernel launches on the caller's stream.  Declarations and contracts are in
// include/fp8q.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fp8q.h"
#include "rollout.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Largest size or leading dimension taken: products of two of them, in elements of up to four
// bytes, stay below 2^63.
constexpr int64_t kMaxDim = 0x7fffffff;
bool dims_ok(int64_t a, int64_t b, int64_t c = 1, int64_t d = 1, int64_t e = 1) {
  return a <= kMaxDim && b <= kMaxDim && c <= kMaxDim && d <= kMaxDim && e <= kMaxDim;
}

// Most tokens, and most workgroups of up to 256 threads in a launch (1024 threads a row: below
// 2^32 threads).
constexpr int64_t kMaxRows = ((int64_t)1 << 22) - 1;
constexpr int64_t kMaxGroups = ((int64_t)1 << 23);

fp8q_status from_hip(hipError_t e) { return e == hipSuccess ? FP8Q_OK : FP8Q_ERR_HIP; }

hipStream_t stream_of(struct ihipStream_t* s) { return reinterpret_cast<hipStream_t>(s); }

bool known(fp8q_dtype d) { return d == FP8Q_BF16 || d == FP8Q_F32; }

// Sizes and alignment of MXFP4 rows.
fp8q_status mx4_rows(const void* codes, int64_t ldc, const void* scales, int64_t rows, int64_t cols) {
  if (!codes || !scales || rows <= 0 || cols <= 0) return FP8Q_ERR_INVAL;
  if (!dims_ok(rows, cols, ldc)) return FP8Q_ERR_UNSUPPORTED;
  if (ldc < fp8q::mx4_padded(cols) / 2) return FP8Q_ERR_INVAL;
  if ((rows + 31) / 32 * ((cols + 511) / 512) > kMaxGroups) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(codes, 16) || ldc % 16 || !aligned(scales, 8)) return FP8Q_ERR_ALIGN;
  return FP8Q_OK;
}

}  // namespace

extern "C" {

fp8q_status fp8q_quantize_mx4(const void* x, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes, int64_t ldc,
                              uint8_t* scales, struct ihipStream_t* stream) {
  if (!x || (cols > 0 && ldx < cols)) return FP8Q_ERR_INVAL;
  const fp8q_status st = mx4_rows(codes, ldc, scales, rows, cols);
  if (st != FP8Q_OK) return st;
  if (ldx > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(x, 2)) return FP8Q_ERR_ALIGN;
  fp8q::Mx4Args a;
  a.x = static_cast<const uint16_t*>(x);
  a.rows = rows;
  a.cols = cols;
  a.ldx = ldx;
  a.codes = codes;
  a.ldc = ldc;
  a.scales = scales;
  return from_hip(fp8q::launch_quantize_mx4(a, stream_of(stream)));
}

fp8q_status fp8q_dequantize_mx4(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t rows, int64_t cols,
                                void* y, int64_t ldy, struct ihipStream_t* stream) {
  if (!y || (cols > 0 && ldy < cols)) return FP8Q_ERR_INVAL;
  const fp8q_status st = mx4_rows(codes, ldc, scales, rows, cols);
  if (st != FP8Q_OK) return st;
  if (ldy > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(y, 2)) return FP8Q_ERR_ALIGN;
  fp8q::Mx4ValuesArgs a;
  a.codes = codes;
  a.scales = scales;
  a.rows = rows;
  a.cols = cols;
  a.ldc = ldc;
  a.y = static_cast<uint16_t*>(y);
  a.ldy = ldy;
  return from_hip(fp8q::launch_dequantize_mx4(a, stream_of(stream)));
}

fp8q_status fp8q_gemm_mx4(const uint8_t* A, const uint8_t* sA, int64_t lda, const uint8_t* B, const uint8_t* sB,
                          int64_t ldb, int64_t M, int64_t N, int64_t K, void* C, int64_t ldc,
                          struct ihipStream_t* stream) {
  if (!A || !sA || !B || !sB || !C) return FP8Q_ERR_INVAL;
  if (M <= 0 || N <= 0 || K <= 0 || lda < K / 2 || ldb < K / 2 || ldc < N) return FP8Q_ERR_INVAL;
  if (!dims_ok(M, N, lda, ldb, ldc) || K > kMaxDim || K % fp8q::kMxPiece) return FP8Q_ERR_UNSUPPORTED;
  // the kernels' 32-bit offsets into the scales and a band of rows, their tile counts
  const int64_t lim = (int64_t)1 << 31;
  if (M * (K / 32) >= lim || N * (K / 32) >= lim) return FP8Q_ERR_UNSUPPORTED;
  if (256 * lda >= lim || 256 * 2 * ldc >= lim || 2048 * ldb >= lim) return FP8Q_ERR_UNSUPPORTED;
  if (((M + 127) / 128) * ((N + 127) / 128) > ((int64_t)1 << 22)) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(A, 16) || !aligned(B, 16) || lda % 16 || ldb % 16 || !aligned(sA, 8) || !aligned(sB, 8) ||
      !aligned(C, 8) || ldc % 4)
    return FP8Q_ERR_ALIGN;
  fp8q::GemmArgs g;
  g.A = A;
  g.B = B;
  g.sA = reinterpret_cast<const float*>(sA);
  g.sB = reinterpret_cast<const float*>(sB);
  g.C = static_cast<uint16_t*>(C);
  g.M = M;
  g.N = N;
  g.K = K / 2;
  g.lda = lda;
  g.ldb = ldb;
  g.ldc = ldc;
  g.sa_ld = 2 * M;
  g.sb_ld = 2 * N;
  g.sa_count = 2 * M * (K / fp8q::kMxPiece);
  g.sb_count = 2 * N * (K / fp8q::kMxPiece);
  g.c_aligned16 = aligned(C, 16) && ldc % 8 == 0;
  g.Cq = nullptr;
  g.Cs = nullptr;
  g.ldq = 0;
  g.cs_ld = 0;
  return from_hip(fp8q::launch_gemm_mx4(g, stream_of(stream)));
}

fp8q_status fp8q_embedding(const void* weight, fp8q_dtype dtype, int64_t V, int64_t C, int64_t ldw,
                           const int64_t* tokens, int64_t T, double scale, void* y, int64_t ldy,
                           struct ihipStream_t* stream) {
  if (!weight || !tokens || !y || !known(dtype)) return FP8Q_ERR_INVAL;
  if (V <= 0 || C <= 0 || T <= 0 || ldw < C || ldy < C || !isfinite((float)scale)) return FP8Q_ERR_INVAL;
  if (T > kMaxRows || C % 16 || !dims_ok(V, C, ldw, ldy) || (T + 3) / 4 * ((C + 2047) / 2048) > kMaxGroups)
    return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(weight, 16) || !aligned(y, 16) || !aligned(tokens, 8) || ldy % 8 || ldw % (dtype == FP8Q_F32 ? 4 : 8))
    return FP8Q_ERR_ALIGN;
  fp8q::EmbeddingArgs a;
  a.weight = weight;
  a.f32 = dtype == FP8Q_F32;
  a.V = V;
  a.C = C;
  a.ldw = ldw;
  a.T = T;
  a.tokens = tokens;
  a.scale = (float)scale;
  a.y = static_cast<uint16_t*>(y);
  a.ldy = ldy;
  return from_hip(fp8q::launch_embedding(a, stream_of(stream)));
}

int64_t fp8q_embedding_backward_workspace(int64_t T, int64_t V, int64_t C) {
  if (T <= 0 || V <= 0 || C <= 0 || T > kMaxRows || !dims_ok(V, C) || C % 16 || V * C >= ((int64_t)1 << 33)) return -1;
  // (launches of less than 2^32 threads: a thread of the zeros 16 bytes, a workgroup of the sums eight
  // tokens or more by a band of 2048 columns; of one token only where that is less, too, see takes_few)
  if (T * ((C + 2047) / 2048) > ((int64_t)1 << 25)) return -1;
  return fp8q::embedding_backward_workspace(T, V, C);
}

fp8q_status fp8q_embedding_backward(const void* dy, int64_t lddy, const int64_t* tokens, int64_t T, int64_t V,
                                    int64_t C, double scale, unsigned flags, void* dweight, fp8q_dtype dtype,
                                    int64_t ldw, void* workspace, int64_t workspace_bytes,
                                    struct ihipStream_t* stream) {
  if (!dy || !tokens || !dweight || !known(dtype) || (flags & ~(unsigned)FP8Q_ACCUMULATE)) return FP8Q_ERR_INVAL;
  if (V <= 0 || C <= 0 || T <= 0 || lddy < C || ldw < C || !isfinite((float)scale)) return FP8Q_ERR_INVAL;
  const int64_t need = fp8q_embedding_backward_workspace(T, V, C);
  if (need < 0 || !dims_ok(lddy, ldw)) return FP8Q_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < need) return FP8Q_ERR_INVAL;
  if (!aligned(dy, 16) || !aligned(dweight, 16) || !aligned(tokens, 8) || !aligned(workspace, 16) || lddy % 8 ||
      ldw % (dtype == FP8Q_F32 ? 4 : 8))
    return FP8Q_ERR_ALIGN;
  fp8q::EmbeddingBackwardArgs a;
  a.dy = static_cast<const uint16_t*>(dy);
  a.T = T;
  a.V = V;
  a.C = C;
  a.lddy = lddy;
  a.tokens = tokens;
  a.scale = (float)scale;
  a.accumulate = (flags & FP8Q_ACCUMULATE) != 0;
  a.f32 = dtype == FP8Q_F32;
  a.dweight = dweight;
  a.ldw = ldw;
  a.workspace = static_cast<uint8_t*>(workspace);
  return from_hip(fp8q::launch_embedding_backward(a, stream_of(stream)));
}

int64_t fp8q_top_logprobs_workspace(int64_t T, int64_t V, int64_t k) {
  if (T <= 0 || V <= 0 || T > kMaxRows || V > kMaxDim || k < 1 || k > FP8Q_MAX_TOP || k > V) return -1;
  return fp8q::top_logprobs_workspace(T, V);
}

fp8q_status fp8q_top_logprobs(const void* logits, fp8q_dtype dtype, int64_t T, int64_t V, int64_t ld,
                              const int64_t* tokens, int64_t k, double temperature, float* logp, float* entropy,
                              int64_t* ids, float* top, void* workspace, int64_t workspace_bytes,
                              struct ihipStream_t* stream) {
  if (!logits || !tokens || !logp || !entropy || !ids || !top || !known(dtype)) return FP8Q_ERR_INVAL;
  const float inverse = (float)(1.0 / temperature);  // (the kernels take log2(e) times it)
  if (T <= 0 || V <= 0 || ld < V || !(temperature > 0.0) || !isfinite(1.5f * inverse) || inverse == 0.0f)
    return FP8Q_ERR_INVAL;
  if (k < 1 || k > FP8Q_MAX_TOP || k > V) return FP8Q_ERR_INVAL;
  if (T > kMaxRows || !dims_ok(T, V, ld)) return FP8Q_ERR_UNSUPPORTED;
  const int64_t need = fp8q_top_logprobs_workspace(T, V, k);
  if (need > 0 && (!workspace || workspace_bytes < need)) return FP8Q_ERR_INVAL;
  if (!aligned(logits, dtype == FP8Q_F32 ? 4 : 2) || !aligned(tokens, 8) || !aligned(logp, 4) || !aligned(entropy, 4) ||
      !aligned(ids, 8) || !aligned(top, 4) || (need > 0 && !aligned(workspace, 16)))
    return FP8Q_ERR_ALIGN;
  fp8q::TopArgs a{};
  a.logits = logits;
  a.f32 = dtype == FP8Q_F32;
  a.T = T;
  a.V = V;
  a.ld = ld;
  a.tokens = tokens;
  a.inv_temperature = inverse;
  a.logp = logp;
  a.entropy = entropy;
  a.k = (int)k;
  a.ids = ids;
  a.top = top;
  a.workspace = static_cast<uint8_t*>(workspace);
  return from_hip(fp8q::launch_top_logprobs(a, stream_of(stream)));
}

}  // extern "C"
