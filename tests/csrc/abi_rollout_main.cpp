// Test driver for a host-only build of abi_rollout.hip, its launchers replaced by the
// recording stubs below, under AddressSanitizer and UndefinedBehaviorSanitizer: every entry
// point with arguments that must be refused, absurd sizes included, and with valid ones.
// Pointers are never dereferenced.  Exit status 0 when every check holds.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "fp8q.h"
#include "rollout.h"

namespace fp8q {
static int launches = 0;
static GemmArgs last_gemm;
static EmbeddingBackwardArgs last_backward;
static TopArgs last_top;
hipError_t launch_quantize_mx4(const Mx4Args&, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_dequantize_mx4(const Mx4ValuesArgs&, hipStream_t) { return ++launches, hipErrorInvalidValue; }
hipError_t launch_gemm_mx4(const GemmArgs& g, hipStream_t) { return ++launches, last_gemm = g, hipSuccess; }
hipError_t launch_embedding(const EmbeddingArgs&, hipStream_t) { return ++launches, hipSuccess; }
int64_t embedding_backward_workspace(int64_t T, int64_t, int64_t C) { return T * C; }
hipError_t launch_embedding_backward(const EmbeddingBackwardArgs& a, hipStream_t) {
  return ++launches, last_backward = a, hipSuccess;
}
int64_t top_logprobs_workspace(int64_t T, int64_t) { return T < 100 ? 16 * T : 0; }
hipError_t launch_top_logprobs(const TopArgs& a, hipStream_t) { return ++launches, last_top = a, hipSuccess; }
}  // namespace fp8q

static int failures = 0;

#define EXPECT(call, want, n)                                                                                  \
  do {                                                                                                         \
    const int before = fp8q::launches;                                                                         \
    const long got = (long)(call);                                                                             \
    if (got != (long)(want) || fp8q::launches - before != (n)) {                                               \
      fprintf(stderr, "line %d: %s -> %ld (want %ld), %d launches\n", __LINE__, #call, got, (long)(want),      \
              fp8q::launches - before);                                                                        \
      ++failures;                                                                                              \
    }                                                                                                          \
  } while (0)

template <typename T>
static T* at(uintptr_t off = 0) {
  return reinterpret_cast<T*>(static_cast<uintptr_t>(0x10000) + off);
}

static const int64_t BIG = INT64_MAX, MOST = 0x7fffffff;

static fp8q_status quant(const void* x = at<void>(), int64_t rows = 4, int64_t cols = 300, int64_t ldx = 300,
                         uint8_t* codes = at<uint8_t>(), int64_t ldc = 256, uint8_t* scales = at<uint8_t>()) {
  return fp8q_quantize_mx4(x, rows, cols, ldx, codes, ldc, scales, nullptr);
}

static fp8q_status values(int64_t cols = 300, void* y = at<void>(), int64_t ldy = 300, int64_t ldc = 256,
                          const uint8_t* scales = at<uint8_t>(), int64_t rows = 4) {
  return fp8q_dequantize_mx4(at<uint8_t>(), ldc, scales, rows, cols, y, ldy, nullptr);
}

static fp8q_status gemm(int64_t M = 4, int64_t N = 12, int64_t K = 512, int64_t lda = 256, int64_t ldb = 256,
                        void* C = at<void>(), int64_t ldc = 12, const uint8_t* A = at<uint8_t>(),
                        const uint8_t* sB = at<uint8_t>()) {
  return fp8q_gemm_mx4(A, at<uint8_t>(), lda, at<uint8_t>(), sB, ldb, M, N, K, C, ldc, nullptr);
}

static fp8q_status embed(int64_t T = 5, int64_t V = 9, int64_t C = 32, int64_t ldw = 32, int64_t ldy = 32,
                         double scale = 1.0, fp8q_dtype t = FP8Q_BF16, const void* w = at<void>(),
                         const int64_t* tokens = at<int64_t>()) {
  return fp8q_embedding(w, t, V, C, ldw, tokens, T, scale, at<void>(), ldy, nullptr);
}

static fp8q_status back(int64_t T = 5, int64_t V = 9, int64_t C = 32, int64_t lddy = 32, int64_t ldw = 32,
                        unsigned flags = 0, fp8q_dtype t = FP8Q_F32, int64_t bytes = 1 << 20, void* ws = at<void>(),
                        double scale = 1.0, void* dw = at<void>()) {
  return fp8q_embedding_backward(at<void>(), lddy, at<int64_t>(), T, V, C, scale, flags, dw, t, ldw, ws, bytes, nullptr);
}

static fp8q_status top(int64_t T = 5, int64_t V = 100, int64_t k = 3, int64_t ld = 100, double t = 1.0,
                       int64_t bytes = 1 << 20, void* ws = at<void>(), fp8q_dtype d = FP8Q_BF16,
                       int64_t* ids = at<int64_t>(), const void* x = at<void>()) {
  return fp8q_top_logprobs(x, d, T, V, ld, at<int64_t>(), k, t, at<float>(), at<float>(), ids, at<float>(), ws, bytes,
                           nullptr);
}

int main() {
  EXPECT(quant(), FP8Q_OK, 1);
  EXPECT(quant(at<void>(2), 4, 299, 301), FP8Q_OK, 1);  // any columns, any even address
  EXPECT(quant(nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(quant(at<void>(1)), FP8Q_ERR_ALIGN, 0);
  EXPECT(quant(at<void>(), 0), FP8Q_ERR_INVAL, 0);
  EXPECT(quant(at<void>(), 4, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(quant(at<void>(), 4, 300, 299), FP8Q_ERR_INVAL, 0);
  EXPECT(quant(at<void>(), 4, 300, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(quant(at<void>(), BIG, BIG, BIG, at<uint8_t>(), BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(quant(at<void>(), MOST, MOST, MOST, at<uint8_t>(), MOST), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(quant(at<void>(), 32 << 23, 512, 512), FP8Q_OK, 1);
  EXPECT(quant(at<void>(), (32 << 23) + 1, 512, 512), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(quant(at<void>(), 4, 300, 300, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(quant(at<void>(), 4, 300, 300, at<uint8_t>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(quant(at<void>(), 4, 300, 300, at<uint8_t>(), 240), FP8Q_ERR_INVAL, 0);  // the rows' zeros have no room
  EXPECT(quant(at<void>(), 4, 300, 300, at<uint8_t>(), 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(quant(at<void>(), 4, 300, 300, at<uint8_t>(), 256, at<uint8_t>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(quant(at<void>(), 4, 300, 300, at<uint8_t>(), 256, nullptr), FP8Q_ERR_INVAL, 0);

  EXPECT(values(), FP8Q_ERR_HIP, 1);  // (its stub fails)
  EXPECT(values(513), FP8Q_ERR_INVAL, 0);
  EXPECT(values(300, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(values(300, at<void>(1)), FP8Q_ERR_ALIGN, 0);
  EXPECT(values(300, at<void>(), 299), FP8Q_ERR_INVAL, 0);
  EXPECT(values(300, at<void>(), BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(values(300, at<void>(), 300, 256, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(values(300, at<void>(), 300, 256, at<uint8_t>(), -1), FP8Q_ERR_INVAL, 0);

  EXPECT(gemm(), FP8Q_OK, 1);
  EXPECT(fp8q::last_gemm.K == 256 && fp8q::last_gemm.sa_ld == 8 && fp8q::last_gemm.sa_count == 16 &&
                 fp8q::last_gemm.sb_count == 48 && !fp8q::last_gemm.c_aligned16 ? 0 : 1, 0, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(), 16), FP8Q_OK, 1);
  EXPECT(fp8q::last_gemm.c_aligned16, 1, 0);
  EXPECT(gemm(0), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 12, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 12, 384), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gemm(4, 12, 512, 240), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 12, 512, 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(gemm(4, 12, 512, 256, 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(), 11), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(), 14), FP8Q_ERR_ALIGN, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(), 12, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(), 12, at<uint8_t>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(gemm(4, 12, 512, 256, 256, at<void>(), 12, at<uint8_t>(), at<uint8_t>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(gemm(BIG, BIG, BIG, BIG, BIG, at<void>(), BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gemm((int64_t)1 << 28, 12, 512), FP8Q_ERR_UNSUPPORTED, 0);             // its scale bytes
  EXPECT(gemm(4, 12, 512, (int64_t)1 << 23), FP8Q_ERR_UNSUPPORTED, 0);          // 256 rows of 2^31 bytes
  EXPECT(gemm(4, 12, 512, 256, (int64_t)1 << 20), FP8Q_ERR_UNSUPPORTED, 0);     // 2048 rows of them
  EXPECT(gemm((int64_t)1 << 20, (int64_t)1 << 20, 512, 256, 256, at<void>(), (int64_t)1 << 20), FP8Q_ERR_UNSUPPORTED, 0);

  EXPECT(embed(), FP8Q_OK, 1);
  EXPECT(embed(5, 9, 32, 36, 32, 1.0, FP8Q_F32), FP8Q_OK, 1);
  EXPECT(embed(5, 9, 32, 36), FP8Q_ERR_ALIGN, 0);
  EXPECT(embed(0), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 9, 40, 40, 40), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(embed(5, 9, 32, 31), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 9, 32, 32, 36), FP8Q_ERR_ALIGN, 0);
  EXPECT(embed(5, 9, 32, 32, 32, NAN), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 9, 32, 32, 32, 1e39), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 9, 32, 32, 32, 1.0, (fp8q_dtype)2), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 9, 32, 32, 32, 1.0, FP8Q_BF16, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(embed(5, 9, 32, 32, 32, 1.0, FP8Q_BF16, at<void>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(embed(5, 9, 32, 32, 32, 1.0, FP8Q_BF16, at<void>(), at<int64_t>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(embed(1 << 22), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(embed(BIG, BIG, BIG, BIG, BIG), FP8Q_ERR_UNSUPPORTED, 0);

  EXPECT(back(), FP8Q_OK, 1);
  EXPECT(fp8q::last_backward.accumulate == 0 && fp8q::last_backward.f32 == 1 ? 0 : 1, 0, 0);
  EXPECT(back(5, 9, 32, 32, 32, FP8Q_ACCUMULATE, FP8Q_BF16), FP8Q_OK, 1);
  EXPECT(fp8q::last_backward.accumulate == 1 && fp8q::last_backward.f32 == 0 ? 0 : 1, 0, 0);
  EXPECT(back(5, 9, 32, 32, 32, 1), FP8Q_ERR_INVAL, 0);
  EXPECT(back(0), FP8Q_ERR_INVAL, 0);
  EXPECT(back(5, 9, 40, 40, 40), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(back(5, 9, 32, 31), FP8Q_ERR_INVAL, 0);
  EXPECT(back(5, 9, 32, 36), FP8Q_ERR_ALIGN, 0);
  EXPECT(back(5, 9, 32, 32, 34), FP8Q_ERR_ALIGN, 0);
  EXPECT(back(5, 9, 32, 32, 36), FP8Q_OK, 1);
  EXPECT(back(5, 9, 32, 32, 36, 0, FP8Q_BF16), FP8Q_ERR_ALIGN, 0);
  EXPECT(back(5, 9, 32, 32, 32, 0, (fp8q_dtype)7), FP8Q_ERR_INVAL, 0);
  EXPECT(back(5, 9, 32, 32, 32, 0, FP8Q_F32, 159), FP8Q_ERR_INVAL, 0);
  EXPECT(back(5, 9, 32, 32, 32, 0, FP8Q_F32, 160), FP8Q_OK, 1);
  EXPECT(back(5, 9, 32, 32, 32, 0, FP8Q_F32, 1 << 20, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(back(5, 9, 32, 32, 32, 0, FP8Q_F32, 1 << 20, at<void>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(back(5, 9, 32, 32, 32, 0, FP8Q_F32, 1 << 20, at<void>(), INFINITY), FP8Q_ERR_INVAL, 0);
  EXPECT(back(5, 9, 32, 32, 32, 0, FP8Q_F32, 1 << 20, at<void>(), 1.0, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(back(1 << 22, 9, 32, 32, 32, 0, FP8Q_F32, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(back(BIG, BIG, BIG, BIG, BIG, 0, FP8Q_F32, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(fp8q_embedding_backward_workspace(5, (int64_t)1 << 29, 16), -1, 0);
  EXPECT(fp8q_embedding_backward_workspace(5, ((int64_t)1 << 29) - 1, 16), 80, 0);
  EXPECT(fp8q_embedding_backward_workspace(1 << 21, 9, 65536), -1, 0);
  EXPECT(fp8q_embedding_backward_workspace(0, 9, 32), -1, 0);

  EXPECT(top(), FP8Q_OK, 1);
  EXPECT(fp8q::last_top.k == 3 && fp8q::last_top.inv_temperature == 1.0f && fp8q::last_top.V == 100 ? 0 : 1, 0, 0);
  EXPECT(top(200, 100, 3, 100, 1.0, 0, nullptr), FP8Q_OK, 1);  // (needs no workspace)
  EXPECT(top(5, 100, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(top(5, 100, 65), FP8Q_ERR_INVAL, 0);
  EXPECT(top(5, 3, 4), FP8Q_ERR_INVAL, 0);
  EXPECT(top(0), FP8Q_ERR_INVAL, 0);
  EXPECT(top(5, 100, 3, 99), FP8Q_ERR_INVAL, 0);
  EXPECT(top(1 << 22), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(top(BIG, BIG, 3, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 79), FP8Q_ERR_INVAL, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 80), FP8Q_OK, 1);
  EXPECT(top(5, 100, 3, 100, 1.0, 1 << 20, at<void>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 1 << 20, at<void>(), (fp8q_dtype)3), FP8Q_ERR_INVAL, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 1 << 20, at<void>(), FP8Q_BF16, at<int64_t>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 1 << 20, at<void>(), FP8Q_BF16, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 1 << 20, at<void>(), FP8Q_F32, at<int64_t>(), at<void>(2)), FP8Q_ERR_ALIGN, 0);
  EXPECT(top(5, 100, 3, 100, 1.0, 1 << 20, at<void>(), FP8Q_BF16, at<int64_t>(), at<void>(2)), FP8Q_OK, 1);
  const double bad_temperatures[] = {0.0, -1.0, (double)NAN, (double)INFINITY, 1e-60, 1e60, 3.5e-39};
  for (double t : bad_temperatures) EXPECT(top(5, 100, 3, 100, t), FP8Q_ERR_INVAL, 0);
  EXPECT(fp8q_top_logprobs_workspace(5, 100, 3), 80, 0);
  EXPECT(fp8q_top_logprobs_workspace(5, 100, 101), -1, 0);
  EXPECT(fp8q_top_logprobs_workspace(BIG, 100, 3), -1, 0);
  printf("%d failures\n", failures);
  return failures != 0;
}
