// Internal interface between the C-ABI layer and the launchers of the
// operators around the FP8 linear layers (norm.hip, gated.hip, requantize.hip,
// loss.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8q.h"
#include "internal.h"

namespace fp8q {

// What a norm writes: y in bf16, or its codes with a scale per row or per
// 1x128 block.
enum NormOut { kNormBf16, kNormRow, kNormBlock };

constexpr int64_t kMaxNormCols = 32768;  // a row is held in registers

struct NormArgs {
  const uint16_t *x, *residual;  // bf16; residual null: h is x
  const void* weight;            // [cols] bf16, or fp32 with weight_f32
  int weight_f32, pow2;
  int64_t rows, cols, ldx, ldr;
  float eps;
  uint16_t* h;                   // x + residual (null without a residual)
  int64_t ldh;
  float* rstd;
  uint16_t* y;
  int64_t ldy;
  uint8_t* codes;
  int64_t ldc;
  float* scales;
};
hipError_t launch_rmsnorm(const NormArgs& a, NormOut out, hipStream_t s);

struct NormBackwardArgs {
  const uint16_t *dy, *h, *dres;  // dres may be null
  const float* rstd;
  const void* weight;
  int weight_f32;
  int64_t rows, cols, lddy, ldh, ldres;
  uint16_t* dx;
  int64_t lddx;
  float* dweight;
  float* partials;  // [norm_backward_groups(rows, cols)][cols]
};
// Workgroups that sum a part of dweight each.
int64_t norm_backward_groups(int64_t rows, int64_t cols);
hipError_t launch_rmsnorm_backward(const NormBackwardArgs& a, hipStream_t s);

// The gated GEMM: GemmArgs with B the gate's rows followed by the up
// projection's (N = 2 F), C the output H [M][ldc] of F columns.
struct GatedArgs : GemmArgs {
  uint16_t* pre = nullptr;  // bf16 [M][ldp]: gate | up, or null
  int64_t ldp = 0;
  int pre_aligned16 = 0;
};
// Quantized output of some sizes is made from H in bf16 (gated_needs_bf16): then C
// is a workspace of M x F for it.
bool gated_needs_bf16(int64_t M, int64_t F, int64_t K);
hipError_t launch_gemm_gated(const GatedArgs& g, bool quantized, hipStream_t s);

struct GatedBackwardArgs {
  const uint16_t *dh, *pre;  // [M][lddh], [M][ldp]
  int64_t M, F, lddh, ldp;
  int pow2, e5m2;
  uint8_t *codes_r, *codes_t;  // [M][ldr], [2 F][ldt]
  int64_t ldr, ldt;
  float *scales_r, *scales_t;
};
hipError_t launch_gated_backward(const GatedBackwardArgs& a, hipStream_t s);

struct RequantArgs {
  const uint8_t* codes;  // E4M3 [rows][ldc]
  const float* scales;   // [cols / 128][rows]
  int64_t rows, cols, ldc;
  int pow2;
  uint8_t* codes_t;      // [cols][ldt]
  int64_t ldt;
  float* scales_t;       // [ceil(rows / 128)][cols]
};
hipError_t launch_requantize_transposed(const RequantArgs& a, hipStream_t s);

// One row of logits a token.  Without dlogits the log-probabilities alone
// (then only logits, tokens, temperature, logp and entropy are read).
struct LossArgs {
  const void* logits;
  int f32;
  int64_t T, V, ld;
  const int64_t* tokens;
  const float *logp_old, *adv, *weight, *w_tis, *logp_ref;  // the last two may be null
  const fp8q_clip_result* clip;  // null: clip_low, clip_high
  float clip_low, clip_high, beta, inv_temperature;
  float* loss;
  void* dlogits;
  int64_t ldd;
  float *logp, *entropy;
  float* terms;     // [T]: each token's part of the loss
  float* partials;  // [T][kLossParts][4], for rows that are split
};
constexpr int kLossParts = 64;  // workgroups that share a row, at most
constexpr int64_t kLossSplitRows = 128;  // only rows fewer than this are split (see split_rows)
// The single element of thread t of a row's workgroup, or -1: of a row of V logits whose
// aligned 16-byte pieces, of n logits each, are `full` from element `head` on, the
// elements before them are those of threads 0 .., the ones after them those of threads
// 32 ...  (V is up to 2^31 - 1: no index is formed past it.)
constexpr int row_edge(int t, int V, int head, int full, int n) {
  if (t < head) return t;
  const int end = head + full * n, after = t - 32;
  return after >= 0 && after < V - end ? end + after : -1;
}

hipError_t launch_logprobs(const LossArgs& a, hipStream_t s);
hipError_t launch_policy_loss(const LossArgs& a, hipStream_t s);

}  // namespace fp8q
