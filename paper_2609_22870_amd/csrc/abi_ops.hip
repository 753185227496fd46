// C-ABI of the operators around the FP8 linear layers: argument validation, then
// kernel launches on the caller's stream.  Declarations and contracts are in
// include/fp8q.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fp8q.h"
#include "ops.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Largest size or leading dimension taken: products of two of them, in
// elements of up to four bytes, stay below 2^63.
constexpr int64_t kMaxDim = 0x7fffffff;
bool dims_ok(int64_t a, int64_t b, int64_t c = 1, int64_t d = 1, int64_t e = 1, int64_t f = 1) {
  return a <= kMaxDim && b <= kMaxDim && c <= kMaxDim && d <= kMaxDim && e <= kMaxDim && f <= kMaxDim;
}

// Most rows of a norm or tokens of a loss: workgroups of up to 1024 threads, one
// a row, stay below 2^32 threads a launch.
constexpr int64_t kMaxRows = ((int64_t)1 << 22) - 1;

// Most 128 x 128 tiles of the backward operands: workgroups of up to 512 threads.
constexpr int64_t kMaxTiles = ((int64_t)1 << 23) - 1;

fp8q_status from_hip(hipError_t e) { return e == hipSuccess ? FP8Q_OK : FP8Q_ERR_HIP; }

hipStream_t stream_of(struct ihipStream_t* s) { return reinterpret_cast<hipStream_t>(s); }

// The checks that both forward norms share, then the kernel arguments but for y.
fp8q_status norm_args(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, unsigned flags,
                      unsigned known, int64_t rows, int64_t cols, float eps, void* h, int64_t ldh, float* rstd,
                      fp8q::NormArgs& a) {
  if (!x || !weight || !rstd || !residual != !h) return FP8Q_ERR_INVAL;
  if ((flags & ~known) || rows <= 0 || cols <= 0 || ldx < cols || !(eps >= 0.0f)) return FP8Q_ERR_INVAL;
  if (residual && (ldr < cols || ldh < cols)) return FP8Q_ERR_INVAL;
  if (rows > kMaxRows || !dims_ok(rows, cols, ldx, residual ? ldr : 1, residual ? ldh : 1)) return FP8Q_ERR_UNSUPPORTED;
  if (cols % 16 || cols > fp8q::kMaxNormCols) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(x, 16) || !aligned(weight, 16) || !aligned(rstd, 4) || ldx % 8) return FP8Q_ERR_ALIGN;
  if (residual && (!aligned(residual, 16) || !aligned(h, 16) || ldr % 8 || ldh % 8)) return FP8Q_ERR_ALIGN;
  a = fp8q::NormArgs{};
  a.x = static_cast<const uint16_t*>(x);
  a.residual = static_cast<const uint16_t*>(residual);
  a.weight = weight;
  a.weight_f32 = (flags & FP8Q_WEIGHT_F32) != 0;
  a.pow2 = (flags & FP8Q_POW2_SCALE) != 0;
  a.rows = rows;
  a.cols = cols;
  a.ldx = ldx;
  a.ldr = ldr;
  a.eps = eps;
  a.h = static_cast<uint16_t*>(h);
  a.ldh = ldh;
  a.rstd = rstd;
  return FP8Q_OK;
}

// The checks that both gated GEMMs share, then the kernel arguments but for
// the output.
fp8q_status gated_args(const uint8_t* A, const float* sA, int64_t lda, const uint8_t* B, const float* sB, int64_t ldb,
                       int64_t M, int64_t F, int64_t K, void* pre, int64_t ldp, fp8q::GatedArgs& g) {
  if (!A || !sA || !B || !sB) return FP8Q_ERR_INVAL;
  if (M <= 0 || F <= 0 || K <= 0 || lda < K || ldb < K) return FP8Q_ERR_INVAL;
  if (!dims_ok(M, F, lda, ldb)) return FP8Q_ERR_UNSUPPORTED;
  if (pre && ldp < 2 * F) return FP8Q_ERR_INVAL;
  if (pre && ldp > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (K % 128 || F % 128) return FP8Q_ERR_UNSUPPORTED;
  // the kernels' 32-bit offsets into B and the scales, and their tile counts
  if (2 * F * ldb >= ((int64_t)1 << 31) || M * (K / 128) >= ((int64_t)1 << 29)) return FP8Q_ERR_UNSUPPORTED;
  if (((M + 127) / 128) * (F / 64) > ((int64_t)1 << 22) || M > (int64_t)65535 * 128) return FP8Q_ERR_UNSUPPORTED;
  if (M * lda >= ((int64_t)1 << 31) && 256 * lda >= ((int64_t)1 << 31)) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(A, 16) || !aligned(B, 16) || lda % 16 || ldb % 16 || !aligned(sA, 4) || !aligned(sB, 4))
    return FP8Q_ERR_ALIGN;
  if (pre && (!aligned(pre, 8) || ldp % 4)) return FP8Q_ERR_ALIGN;
  g.A = A;
  g.B = B;
  g.sA = sA;
  g.sB = sB;
  g.C = nullptr;
  g.M = M;
  g.N = 2 * F;
  g.K = K;
  g.lda = lda;
  g.ldb = ldb;
  g.ldc = 0;
  g.sa_ld = M;
  g.sb_ld = 2 * F;
  g.sa_count = M * (K / 128);
  g.sb_count = (2 * F / 128) * (K / 128);
  g.c_aligned16 = 0;
  g.Cq = nullptr;
  g.Cs = nullptr;
  g.ldq = 0;
  g.cs_ld = 0;
  g.pre = static_cast<uint16_t*>(pre);
  g.ldp = ldp;
  g.pre_aligned16 = pre && aligned(pre, 16) && ldp % 8 == 0;
  return FP8Q_OK;
}

// Workspace of the loss: each token's part of it, then the sums of the parts
// of split rows (a fixed place for each, 16-byte aligned).
int64_t terms_bytes(int64_t T) { return (4 * T + 15) / 16 * 16; }

// The checks that the two calls on logits share, then their kernel arguments.
fp8q_status logit_args(const void* logits, fp8q_dtype dtype, int64_t T, int64_t V, int64_t ld, const int64_t* tokens,
                       double temperature, float* logp, float* entropy, void* workspace, int64_t workspace_bytes,
                       fp8q::LossArgs& a) {
  if (!logits || !tokens || !logp || !entropy || (dtype != FP8Q_BF16 && dtype != FP8Q_F32)) return FP8Q_ERR_INVAL;
  const float inverse = (float)(1.0 / temperature);  // (the kernels take log2(e) times it)
  if (T <= 0 || V <= 0 || ld < V || !(temperature > 0.0) || !isfinite(1.5f * inverse) || inverse == 0.0f)
    return FP8Q_ERR_INVAL;
  if (T > kMaxRows || !dims_ok(T, V, ld)) return FP8Q_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < fp8q_policy_loss_workspace(T, V)) return FP8Q_ERR_INVAL;
  if (!aligned(logits, dtype == FP8Q_F32 ? 4 : 2) || !aligned(tokens, 8) || !aligned(logp, 4) || !aligned(entropy, 4) ||
      !aligned(workspace, 16))
    return FP8Q_ERR_ALIGN;
  a = fp8q::LossArgs{};
  a.logits = logits;
  a.f32 = dtype == FP8Q_F32;
  a.T = T;
  a.V = V;
  a.ld = ld;
  a.tokens = tokens;
  a.inv_temperature = inverse;
  a.logp = logp;
  a.entropy = entropy;
  a.terms = static_cast<float*>(workspace);
  a.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + terms_bytes(T));
  return FP8Q_OK;
}

}  // namespace

extern "C" {

fp8q_status fp8q_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                         unsigned flags, int64_t rows, int64_t cols, float eps, void* h, int64_t ldh, float* rstd,
                         void* y, int64_t ldy, struct ihipStream_t* stream) {
  fp8q::NormArgs a;
  const fp8q_status st =
      norm_args(x, ldx, residual, ldr, weight, flags, FP8Q_WEIGHT_F32, rows, cols, eps, h, ldh, rstd, a);
  if (!y || (rows > 0 && ldy < cols)) return FP8Q_ERR_INVAL;
  if (st != FP8Q_OK) return st;
  if (ldy > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(y, 16) || ldy % 8) return FP8Q_ERR_ALIGN;
  a.y = static_cast<uint16_t*>(y);
  a.ldy = ldy;
  return from_hip(fp8q::launch_rmsnorm(a, fp8q::kNormBf16, stream_of(stream)));
}

fp8q_status fp8q_rmsnorm_quantize(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                                  unsigned flags, int64_t rows, int64_t cols, float eps, void* h, int64_t ldh,
                                  float* rstd, fp8q_granularity g, uint8_t* codes, int64_t ldc, float* scales,
                                  struct ihipStream_t* stream) {
  fp8q::NormArgs a;
  const fp8q_status st = norm_args(x, ldx, residual, ldr, weight, flags, FP8Q_WEIGHT_F32 | FP8Q_POW2_SCALE, rows, cols,
                                   eps, h, ldh, rstd, a);
  if (!codes || !scales || (rows > 0 && ldc < cols) || g < FP8Q_TENSOR || g > FP8Q_BLOCK_128x128) return FP8Q_ERR_INVAL;
  if (st != FP8Q_OK) return st;
  if (ldc > kMaxDim || (g != FP8Q_BLOCK_1x128 && g != FP8Q_ROW)) return FP8Q_ERR_UNSUPPORTED;
  if (g == FP8Q_BLOCK_1x128 && cols % 128) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(codes, 16) || ldc % 16 || !aligned(scales, 4)) return FP8Q_ERR_ALIGN;
  a.codes = codes;
  a.ldc = ldc;
  a.scales = scales;
  return from_hip(fp8q::launch_rmsnorm(a, g == FP8Q_ROW ? fp8q::kNormRow : fp8q::kNormBlock, stream_of(stream)));
}

int64_t fp8q_rmsnorm_backward_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || rows > kMaxRows || cols % 16 || cols > fp8q::kMaxNormCols) return -1;
  return fp8q::norm_backward_groups(rows, cols) * cols * 4;
}

fp8q_status fp8q_rmsnorm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* rstd,
                                  const void* weight, unsigned flags, const void* dres, int64_t ldres, int64_t rows,
                                  int64_t cols, void* dx, int64_t lddx, float* dweight, void* workspace,
                                  int64_t workspace_bytes, struct ihipStream_t* stream) {
  if (!dy || !h || !rstd || !weight || !dx || !dweight) return FP8Q_ERR_INVAL;
  if ((flags & ~(unsigned)FP8Q_WEIGHT_F32) || rows <= 0 || cols <= 0) return FP8Q_ERR_INVAL;
  if (lddy < cols || ldh < cols || lddx < cols || (dres && ldres < cols)) return FP8Q_ERR_INVAL;
  if (rows > kMaxRows || !dims_ok(rows, cols, lddy, ldh, lddx, dres ? ldres : 1)) return FP8Q_ERR_UNSUPPORTED;
  if (cols % 16 || cols > fp8q::kMaxNormCols) return FP8Q_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < fp8q_rmsnorm_backward_workspace(rows, cols)) return FP8Q_ERR_INVAL;
  if (!aligned(dy, 16) || !aligned(h, 16) || !aligned(weight, 16) || !aligned(dx, 16) || !aligned(workspace, 16) ||
      !aligned(rstd, 4) || !aligned(dweight, 4) || lddy % 8 || ldh % 8 || lddx % 8)
    return FP8Q_ERR_ALIGN;
  if (dres && (!aligned(dres, 16) || ldres % 8)) return FP8Q_ERR_ALIGN;
  fp8q::NormBackwardArgs a;
  a.dy = static_cast<const uint16_t*>(dy);
  a.h = static_cast<const uint16_t*>(h);
  a.dres = static_cast<const uint16_t*>(dres);
  a.rstd = rstd;
  a.weight = weight;
  a.weight_f32 = (flags & FP8Q_WEIGHT_F32) != 0;
  a.rows = rows;
  a.cols = cols;
  a.lddy = lddy;
  a.ldh = ldh;
  a.ldres = ldres;
  a.dx = static_cast<uint16_t*>(dx);
  a.lddx = lddx;
  a.dweight = dweight;
  a.partials = static_cast<float*>(workspace);
  return from_hip(fp8q::launch_rmsnorm_backward(a, stream_of(stream)));
}

fp8q_status fp8q_gemm_gated(const uint8_t* A, const float* sA, int64_t lda, const uint8_t* B, const float* sB,
                            int64_t ldb, int64_t M, int64_t F, int64_t K, void* H, int64_t ldh, void* pre, int64_t ldp,
                            struct ihipStream_t* stream) {
  fp8q::GatedArgs g;
  const fp8q_status st = gated_args(A, sA, lda, B, sB, ldb, M, F, K, pre, ldp, g);
  if (!H || (F > 0 && ldh < F)) return FP8Q_ERR_INVAL;
  if (st != FP8Q_OK) return st;
  if (ldh > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(H, 8) || ldh % 4) return FP8Q_ERR_ALIGN;
  g.C = static_cast<uint16_t*>(H);
  g.ldc = ldh;
  g.c_aligned16 = aligned(H, 16) && ldh % 8 == 0;
  return from_hip(fp8q::launch_gemm_gated(g, false, stream_of(stream)));
}

int64_t fp8q_gemm_gated_workspace(int64_t M, int64_t F, int64_t K) {
  if (M <= 0 || F <= 0 || K <= 0 || !dims_ok(M, F, K)) return -1;
  return fp8q::gated_needs_bf16(M, F, K) ? 2 * M * F : 0;
}

fp8q_status fp8q_gemm_gated_quantized(const uint8_t* A, const float* sA, int64_t lda, const uint8_t* B, const float* sB,
                                      int64_t ldb, int64_t M, int64_t F, int64_t K, void* pre, int64_t ldp,
                                      uint8_t* codes, int64_t ldq, float* scales, void* workspace,
                                      int64_t workspace_bytes, struct ihipStream_t* stream) {
  fp8q::GatedArgs g;
  const fp8q_status st = gated_args(A, sA, lda, B, sB, ldb, M, F, K, pre, ldp, g);
  if (!codes || !scales || (F > 0 && ldq < F)) return FP8Q_ERR_INVAL;
  if (st != FP8Q_OK) return st;
  if (ldq > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(codes, 16) || ldq % 16 || !aligned(scales, 4)) return FP8Q_ERR_ALIGN;
  if (const int64_t need = fp8q_gemm_gated_workspace(M, F, K)) {
    if (!workspace || workspace_bytes < need) return FP8Q_ERR_INVAL;
    if (!aligned(workspace, 16)) return FP8Q_ERR_ALIGN;
    g.C = static_cast<uint16_t*>(workspace);
    g.ldc = F;
    g.c_aligned16 = 1;
  }
  g.Cq = codes;
  g.Cs = scales;
  g.ldq = ldq;
  g.cs_ld = M;
  return from_hip(fp8q::launch_gemm_gated(g, true, stream_of(stream)));
}

fp8q_status fp8q_gated_backward(const void* dh, int64_t lddh, const void* pre, int64_t ldp, int64_t M, int64_t F,
                                unsigned flags, uint8_t* codes_r, int64_t ldr, float* scales_r, uint8_t* codes_t,
                                int64_t ldt, float* scales_t, struct ihipStream_t* stream) {
  if (!dh || !pre || !codes_r || !scales_r || !codes_t || !scales_t) return FP8Q_ERR_INVAL;
  if ((flags & ~(unsigned)(FP8Q_POW2_SCALE | FP8Q_E5M2)) || M <= 0 || F <= 0) return FP8Q_ERR_INVAL;
  if (!dims_ok(M, F, lddh, ldp, ldr, ldt)) return FP8Q_ERR_UNSUPPORTED;
  if (lddh < F || ldp < 2 * F || ldr < 2 * F || ldt < (M + 127) / 128 * 128) return FP8Q_ERR_INVAL;
  if (F % 128 || (M + 127) / 128 * (F / 128) > kMaxTiles) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(dh, 16) || !aligned(pre, 16) || !aligned(codes_r, 16) || !aligned(codes_t, 16) || !aligned(scales_r, 4) ||
      !aligned(scales_t, 4) || lddh % 8 || ldp % 8 || ldr % 16 || ldt % 16)
    return FP8Q_ERR_ALIGN;
  fp8q::GatedBackwardArgs a;
  a.dh = static_cast<const uint16_t*>(dh);
  a.pre = static_cast<const uint16_t*>(pre);
  a.M = M;
  a.F = F;
  a.lddh = lddh;
  a.ldp = ldp;
  a.pow2 = (flags & FP8Q_POW2_SCALE) != 0;
  a.e5m2 = (flags & FP8Q_E5M2) != 0;
  a.codes_r = codes_r;
  a.codes_t = codes_t;
  a.ldr = ldr;
  a.ldt = ldt;
  a.scales_r = scales_r;
  a.scales_t = scales_t;
  return from_hip(fp8q::launch_gated_backward(a, stream_of(stream)));
}

fp8q_status fp8q_requantize_transposed(const uint8_t* codes, int64_t ldc, const float* scales, int64_t rows,
                                       int64_t cols, unsigned flags, uint8_t* codes_t, int64_t ldt, float* scales_t,
                                       struct ihipStream_t* stream) {
  if (!codes || !scales || !codes_t || !scales_t) return FP8Q_ERR_INVAL;
  if ((flags & ~(unsigned)FP8Q_POW2_SCALE) || rows <= 0 || cols <= 0) return FP8Q_ERR_INVAL;
  if (!dims_ok(rows, cols, ldc, ldt)) return FP8Q_ERR_UNSUPPORTED;
  if (ldc < cols || ldt < (rows + 127) / 128 * 128) return FP8Q_ERR_INVAL;
  if (cols % 128 || (rows + 127) / 128 * (cols / 128) > kMaxTiles) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(codes, 16) || !aligned(codes_t, 16) || !aligned(scales, 4) || !aligned(scales_t, 4) || ldc % 16 ||
      ldt % 16)
    return FP8Q_ERR_ALIGN;
  fp8q::RequantArgs a;
  a.codes = codes;
  a.scales = scales;
  a.rows = rows;
  a.cols = cols;
  a.ldc = ldc;
  a.pow2 = (flags & FP8Q_POW2_SCALE) != 0;
  a.codes_t = codes_t;
  a.ldt = ldt;
  a.scales_t = scales_t;
  return from_hip(fp8q::launch_requantize_transposed(a, stream_of(stream)));
}

int64_t fp8q_policy_loss_workspace(int64_t T, int64_t V) {
  if (T <= 0 || V <= 0 || T > kMaxRows || V > kMaxDim) return -1;
  const int64_t split = T < fp8q::kLossSplitRows ? T : fp8q::kLossSplitRows;
  return terms_bytes(T) + split * fp8q::kLossParts * 16;
}

fp8q_status fp8q_token_logprobs(const void* logits, fp8q_dtype dtype, int64_t T, int64_t V, int64_t ld,
                                const int64_t* tokens, double temperature, float* logp, float* entropy,
                                void* workspace, int64_t workspace_bytes, struct ihipStream_t* stream) {
  fp8q::LossArgs a;
  const fp8q_status st = logit_args(logits, dtype, T, V, ld, tokens, temperature, logp, entropy, workspace,
                                    workspace_bytes, a);
  if (st != FP8Q_OK) return st;
  return from_hip(fp8q::launch_logprobs(a, stream_of(stream)));
}

fp8q_status fp8q_policy_loss(const void* logits, fp8q_dtype dtype, int64_t T, int64_t V, int64_t ld,
                             const fp8q_policy_batch* batch, float* loss, void* dlogits, int64_t ldd, float* logp,
                             float* entropy, void* workspace, int64_t workspace_bytes, struct ihipStream_t* stream) {
  if (!batch || !loss || !dlogits) return FP8Q_ERR_INVAL;
  const fp8q_policy_batch b = *batch;
  fp8q::LossArgs a;
  const fp8q_status st = logit_args(logits, dtype, T, V, ld, b.tokens, b.temperature, logp, entropy, workspace,
                                    workspace_bytes, a);
  if (!b.logp_old || !b.adv || !b.weight || (V > 0 && ldd < V)) return FP8Q_ERR_INVAL;
  if ((!b.clip && !(b.clip_low <= b.clip_high)) || isnan(b.beta)) return FP8Q_ERR_INVAL;
  if (st != FP8Q_OK) return st;
  if (ldd > kMaxDim) return FP8Q_ERR_UNSUPPORTED;
  if (!aligned(dlogits, dtype == FP8Q_F32 ? 4 : 2) || !aligned(loss, 4) || !aligned(b.logp_old, 4) ||
      !aligned(b.adv, 4) || !aligned(b.weight, 4) || !aligned(b.w_tis, 4) || !aligned(b.logp_ref, 4) ||
      !aligned(b.clip, 8))
    return FP8Q_ERR_ALIGN;
  a.logp_old = b.logp_old;
  a.adv = b.adv;
  a.weight = b.weight;
  a.w_tis = b.w_tis;
  a.logp_ref = (float)b.beta != 0.0f ? b.logp_ref : nullptr;
  a.clip = b.clip;
  a.clip_low = (float)b.clip_low;
  a.clip_high = (float)b.clip_high;
  a.beta = (float)b.beta;
  a.loss = loss;
  a.dlogits = dlogits;
  a.ldd = ldd;
  return from_hip(fp8q::launch_policy_loss(a, stream_of(stream)));
}

}  // extern "C"
