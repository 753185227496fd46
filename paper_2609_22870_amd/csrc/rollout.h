// Internal interface between the C-ABI layer and the launchers of the 4-bit rollout's
// operators and of the two ends of the policy (mx4.hip, gemm_mx4.hip, embedding.hip,
// top.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8q.h"
#include "internal.h"
#include "ops.h"

namespace fp8q {

// MXFP4: rows of codes are filled up to whole pieces of 256, eight scale bytes each.
constexpr int64_t kMxUnit = 32, kMxPiece = 256;
constexpr int64_t mx4_padded(int64_t cols) { return (cols + kMxPiece - 1) / kMxPiece * kMxPiece; }

struct Mx4Args {
  const uint16_t* x;  // bf16 [rows][ldx]
  int64_t rows, cols, ldx;
  uint8_t* codes;     // [rows][ldc] bytes, mx4_padded(cols) / 2 of them a row
  int64_t ldc;
  uint8_t* scales;    // [mx4_padded(cols) / 256][rows][8]
};
hipError_t launch_quantize_mx4(const Mx4Args& a, hipStream_t s);

struct Mx4ValuesArgs {
  const uint8_t *codes, *scales;
  int64_t rows, cols, ldc;
  uint16_t* y;  // bf16 [rows][ldy]
  int64_t ldy;
};
hipError_t launch_dequantize_mx4(const Mx4ValuesArgs& a, hipStream_t s);

// GemmArgs as kPairMx4 has them.
hipError_t launch_gemm_mx4(const GemmArgs& g, hipStream_t s);

struct EmbeddingArgs {
  const void* weight;  // [V][ldw], bf16 or fp32
  int f32;
  int64_t V, C, ldw, T;
  const int64_t* tokens;
  float scale;
  uint16_t* y;  // bf16 [T][ldy]
  int64_t ldy;
};
hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t s);

struct EmbeddingBackwardArgs {
  const uint16_t* dy;  // bf16 [T][lddy]
  int64_t T, V, C, lddy;
  const int64_t* tokens;
  float scale;
  int accumulate, f32;  // f32: dweight's type
  void* dweight;        // [V][ldw]
  int64_t ldw;
  uint8_t* workspace;   // embedding_backward_workspace(T, V, C) bytes
};
int64_t embedding_backward_workspace(int64_t T, int64_t V, int64_t C);
hipError_t launch_embedding_backward(const EmbeddingBackwardArgs& a, hipStream_t s);

struct TopArgs : LossArgs {
  int k;
  int64_t* ids;  // [T][k]
  float* top;    // [T][k]
  uint8_t* workspace;
};
int64_t top_logprobs_workspace(int64_t T, int64_t V);
hipError_t launch_top_logprobs(const TopArgs& a, hipStream_t s);

}  // namespace fp8q
