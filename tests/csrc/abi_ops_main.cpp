// Test driver for a host-only build of the operators' C-ABI (abi_ops.hip, its
// launchers replaced by recording stubs below) under AddressSanitizer and
// UndefinedBehaviorSanitizer: every entry point with arguments that must be
// refused, absurd sizes included, which must return the documented status
// without reaching a launcher, and with valid ones, which must reach one.
// Pointers are never dereferenced.  Exit status 0 when every check holds.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "fp8q.h"
#include "ops.h"

namespace fp8q {
static int launches = 0;
static LossArgs last_loss;
static GatedArgs last_gated;
hipError_t launch_rmsnorm(const NormArgs&, NormOut, hipStream_t) { return ++launches, hipSuccess; }
int64_t norm_backward_groups(int64_t rows, int64_t) { return rows < 512 ? rows : 512; }
hipError_t launch_rmsnorm_backward(const NormBackwardArgs&, hipStream_t) { return ++launches, hipSuccess; }
bool gated_needs_bf16(int64_t M, int64_t, int64_t) { return M < 100; }
hipError_t launch_gemm_gated(const GatedArgs& g, bool, hipStream_t) { return ++launches, last_gated = g, hipSuccess; }
hipError_t launch_gated_backward(const GatedBackwardArgs&, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_requantize_transposed(const RequantArgs&, hipStream_t) { return ++launches, hipErrorInvalidValue; }
hipError_t launch_logprobs(const LossArgs& a, hipStream_t) { return ++launches, last_loss = a, hipSuccess; }
hipError_t launch_policy_loss(const LossArgs& a, hipStream_t) { return ++launches, last_loss = a, hipSuccess; }
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

static const int64_t BIG = INT64_MAX, WIDE = (int64_t)1 << 40;

static fp8q_status norm(const void* x = at<void>(), int64_t ldx = 256, const void* r = at<void>(), int64_t ldr = 256,
                        const void* w = at<void>(), unsigned flags = 0, int64_t rows = 4, int64_t cols = 256,
                        float eps = 1e-6f, void* h = at<void>(), int64_t ldh = 256, float* rstd = at<float>(),
                        void* y = at<void>(), int64_t ldy = 256) {
  return fp8q_rmsnorm(x, ldx, r, ldr, w, flags, rows, cols, eps, h, ldh, rstd, y, ldy, nullptr);
}

static fp8q_status normq(fp8q_granularity g, unsigned flags = 0, int64_t cols = 256, int64_t ldc = 256,
                         uint8_t* codes = at<uint8_t>(), float* scales = at<float>()) {
  return fp8q_rmsnorm_quantize(at<void>(), 256, nullptr, 0, at<void>(), flags, 4, cols, 0.0f, nullptr, 0, at<float>(), g,
                               codes, ldc, scales, nullptr);
}

static fp8q_status normb(int64_t rows = 4, int64_t cols = 256, int64_t ld = 256, void* ws = at<void>(),
                         int64_t bytes = 1 << 20, const void* dres = at<void>(), unsigned flags = 0) {
  return fp8q_rmsnorm_backward(at<void>(), ld, at<void>(), ld, at<float>(), at<void>(), flags, dres, ld, rows, cols,
                               at<void>(), ld, at<float>(), ws, bytes, nullptr);
}

static fp8q_status gated(int64_t M = 200, int64_t F = 256, int64_t K = 256, int64_t lda = 256, int64_t ldb = 256,
                         void* H = at<void>(), int64_t ldh = 256, void* pre = at<void>(), int64_t ldp = 512) {
  return fp8q_gemm_gated(at<uint8_t>(), at<float>(), lda, at<uint8_t>(), at<float>(), ldb, M, F, K, H, ldh, pre, ldp,
                         nullptr);
}

static fp8q_status gatedq(int64_t M, void* ws, int64_t bytes, int64_t ldq = 256, int64_t F = 256) {
  return fp8q_gemm_gated_quantized(at<uint8_t>(), at<float>(), 256, at<uint8_t>(), at<float>(), 256, M, F, 256, nullptr,
                                   0, at<uint8_t>(), ldq, at<float>(), ws, bytes, nullptr);
}

static fp8q_status gatedb(int64_t M = 200, int64_t F = 256, unsigned flags = 0, int64_t lddh = 256, int64_t ldp = 512,
                          int64_t ldr = 512, int64_t ldt = 256) {
  return fp8q_gated_backward(at<void>(), lddh, at<void>(), ldp, M, F, flags, at<uint8_t>(), ldr, at<float>(),
                             at<uint8_t>(), ldt, at<float>(), nullptr);
}

static fp8q_status requant(int64_t rows = 200, int64_t cols = 256, int64_t ldc = 256, int64_t ldt = 256,
                           unsigned flags = 0, uint8_t* out = at<uint8_t>()) {
  return fp8q_requantize_transposed(at<uint8_t>(), ldc, at<float>(), rows, cols, flags, out, ldt, at<float>(), nullptr);
}

static fp8q_policy_batch batch() {
  fp8q_policy_batch b{};
  b.tokens = at<int64_t>();
  b.logp_old = b.adv = b.weight = at<float>();
  b.clip_low = 0.8;
  b.clip_high = 1.2;
  b.temperature = 1.0;
  return b;
}

static fp8q_status loss(const fp8q_policy_batch* b, int64_t T = 8, int64_t V = 1000, int64_t ld = 1000,
                        fp8q_dtype t = FP8Q_BF16, int64_t bytes = 1 << 20, void* dl = at<void>(), int64_t ldd = 1000,
                        void* ws = at<void>()) {
  return fp8q_policy_loss(at<void>(), t, T, V, ld, b, at<float>(), dl, ldd, at<float>(), at<float>(), ws, bytes,
                          nullptr);
}

int main() {
  EXPECT(norm(), FP8Q_OK, 1);
  EXPECT(norm(at<void>(), 256, nullptr, 0, at<void>(), FP8Q_WEIGHT_F32, 4, 256, 0.f, nullptr, 0), FP8Q_OK, 1);
  EXPECT(norm(nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, nullptr), FP8Q_ERR_INVAL, 0);  // h without a residual
  EXPECT(norm(at<void>(), 255), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 255), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 1), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), FP8Q_POW2_SCALE), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), BIG, at<void>(), BIG, at<void>(), 0, BIG, BIG, 1e-6f, at<void>(), BIG, at<float>(),
              at<void>(), BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 1 << 22), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, (1 << 22) - 1), FP8Q_OK, 1);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 248), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(norm(at<void>(), 32784, at<void>(), 32784, at<void>(), 0, 4, 32784, 1e-6f, at<void>(), 32784, at<float>(),
              at<void>(), 32784), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 256, -1.f), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 256, NAN), FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(2)), FP8Q_ERR_ALIGN, 0);
  EXPECT(norm(at<void>(), 260), FP8Q_ERR_ALIGN, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 256, 1e-6f, at<void>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 256, 1e-6f, at<void>(), 256, at<float>(2)),
         FP8Q_ERR_ALIGN, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 256, 1e-6f, at<void>(), 256, at<float>(), nullptr),
         FP8Q_ERR_INVAL, 0);
  EXPECT(norm(at<void>(), 256, at<void>(), 256, at<void>(), 0, 4, 256, 1e-6f, at<void>(), 256, at<float>(), at<void>(),
              WIDE), FP8Q_ERR_UNSUPPORTED, 0);

  EXPECT(normq(FP8Q_BLOCK_1x128), FP8Q_OK, 1);
  EXPECT(normq(FP8Q_ROW, FP8Q_POW2_SCALE | FP8Q_WEIGHT_F32, 144), FP8Q_OK, 1);
  EXPECT(normq(FP8Q_BLOCK_1x128, 0, 144), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(normq(FP8Q_TENSOR), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(normq((fp8q_granularity)9), FP8Q_ERR_INVAL, 0);
  EXPECT(normq(FP8Q_ROW, FP8Q_E5M2), FP8Q_ERR_INVAL, 0);
  EXPECT(normq(FP8Q_ROW, 0, 256, 240), FP8Q_ERR_INVAL, 0);
  EXPECT(normq(FP8Q_ROW, 0, 256, 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(normq(FP8Q_ROW, 0, 256, 256, at<uint8_t>(8)), FP8Q_ERR_ALIGN, 0);
  EXPECT(normq(FP8Q_ROW, 0, 256, 256, at<uint8_t>(), nullptr), FP8Q_ERR_INVAL, 0);

  EXPECT(normb(), FP8Q_OK, 1);
  EXPECT(normb(4, 256, 256, at<void>(), 1 << 20, nullptr), FP8Q_OK, 1);
  EXPECT(normb(4, 256, 256, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(normb(4, 256, 256, at<void>(), 4 * 256 * 4 - 1), FP8Q_ERR_INVAL, 0);
  EXPECT(normb(4, 256, 256, at<void>(), 4 * 256 * 4), FP8Q_OK, 1);
  EXPECT(normb(4, 256, 256, at<void>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(normb(4, 256, 248), FP8Q_ERR_INVAL, 0);
  EXPECT(normb(4, 256, 260), FP8Q_ERR_ALIGN, 0);
  EXPECT(normb(4, 264, 264), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(normb(BIG, 256, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(normb(4, 256, 256, at<void>(), 1 << 20, at<void>(), FP8Q_POW2_SCALE), FP8Q_ERR_INVAL, 0);
  EXPECT(fp8q_rmsnorm_backward_workspace(BIG, 256), -1, 0);
  EXPECT(fp8q_rmsnorm_backward_workspace(4, 255), -1, 0);
  EXPECT(fp8q_rmsnorm_backward_workspace(4, 256), 4096, 0);

  EXPECT(gated(), FP8Q_OK, 1);
  EXPECT(fp8q::last_gated.N == 512 && fp8q::last_gated.sa_count == 400 && fp8q::last_gated.sb_count == 8 ? 0 : 1, 0, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(), 256, nullptr, 0), FP8Q_OK, 1);
  EXPECT(gated(0), FP8Q_ERR_INVAL, 0);
  EXPECT(gated(200, 192), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gated(200, 256, 192), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gated(200, 256, 512), FP8Q_ERR_INVAL, 0);
  EXPECT(gated(BIG, 256, 256), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gated(200, BIG, 256, 256, 256, at<void>(), BIG, nullptr, 0), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gated(200, 256, 256, 256, (int64_t)1 << 22), FP8Q_ERR_UNSUPPORTED, 0);   // 2 F ldb of 2^31
  EXPECT(gated(200, 256, 256, (int64_t)1 << 24), FP8Q_ERR_UNSUPPORTED, 0);        // 256 rows of 2^32 bytes
  EXPECT(gated(9000000, 256), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gated(200, 256, 256, 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(gated(200, 256, 256, 256, 256, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(), 255), FP8Q_ERR_INVAL, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(), 258), FP8Q_ERR_ALIGN, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(4)), FP8Q_ERR_ALIGN, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(), 256, at<void>(), 511), FP8Q_ERR_INVAL, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(), 256, at<void>(), 514), FP8Q_ERR_ALIGN, 0);
  EXPECT(gated(200, 256, 256, 256, 256, at<void>(), 256, at<void>(), WIDE), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gatedq(200, nullptr, 0), FP8Q_OK, 1);
  EXPECT(gatedq(50, nullptr, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(gatedq(50, at<void>(), 2 * 50 * 256 - 1), FP8Q_ERR_INVAL, 0);
  EXPECT(gatedq(50, at<void>(8), 1 << 20), FP8Q_ERR_ALIGN, 0);
  EXPECT(gatedq(50, at<void>(), 2 * 50 * 256), FP8Q_OK, 1);
  EXPECT(gatedq(200, nullptr, 0, 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(gatedq(200, nullptr, 0, 240), FP8Q_ERR_INVAL, 0);
  EXPECT(fp8q_gemm_gated_workspace(50, 256, 256), 2 * 50 * 256, 0);
  EXPECT(fp8q_gemm_gated_workspace(200, 256, 256), 0, 0);
  EXPECT(fp8q_gemm_gated_workspace(BIG, BIG, BIG), -1, 0);

  EXPECT(gatedb(), FP8Q_OK, 1);
  EXPECT(gatedb(200, 256, FP8Q_E5M2 | FP8Q_POW2_SCALE), FP8Q_OK, 1);
  EXPECT(gatedb(200, 256, FP8Q_OUT_TRANSPOSED), FP8Q_ERR_INVAL, 0);
  EXPECT(gatedb(200, 192), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gatedb(BIG, BIG, 0, BIG, BIG, BIG, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(gatedb(257), FP8Q_ERR_INVAL, 0);  // 384 tokens do not fit ldt
  EXPECT(gatedb(200, 256, 0, 255), FP8Q_ERR_INVAL, 0);
  EXPECT(gatedb(200, 256, 0, 260), FP8Q_ERR_ALIGN, 0);
  EXPECT(gatedb(200, 256, 0, 256, 512, 520), FP8Q_ERR_ALIGN, 0);
  EXPECT(gatedb((int64_t)1 << 30, 256, 0, 256, 512, 512, (int64_t)1 << 30), FP8Q_ERR_UNSUPPORTED, 0);

  EXPECT(requant(), FP8Q_ERR_HIP, 1);  // (its stub fails)
  EXPECT(requant(257), FP8Q_ERR_INVAL, 0);
  EXPECT(requant(200, 200), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(requant(200, 256, 256, 256, FP8Q_E5M2), FP8Q_ERR_INVAL, 0);
  EXPECT(requant(BIG, BIG, BIG, BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(requant(200, 256, 264), FP8Q_ERR_ALIGN, 0);
  EXPECT(requant(200, 256, 256, 256, 0, nullptr), FP8Q_ERR_INVAL, 0);

  fp8q_policy_batch b = batch();
  EXPECT(loss(&b), FP8Q_OK, 1);
  EXPECT(fp8q::last_loss.clip_low == 0.8f && fp8q::last_loss.inv_temperature == 1.0f ? 0 : 1, 0, 0);
  b.logp_ref = at<float>();
  EXPECT(loss(&b), FP8Q_OK, 1);  // (no KL term with a coefficient of zero)
  EXPECT(fp8q::last_loss.logp_ref == nullptr ? 0 : 1, 0, 0);
  b.beta = 0.1;
  EXPECT(loss(&b), FP8Q_OK, 1);
  EXPECT(fp8q::last_loss.logp_ref != nullptr ? 0 : 1, 0, 0);
  b = batch();
  EXPECT(loss(nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, 0), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, 8, 1000, 999), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, BIG, BIG, BIG, FP8Q_BF16, BIG, at<void>(), BIG), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(loss(&b, 1 << 22), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(loss(&b, 8, 1000, 1000, (fp8q_dtype)2), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_F32, fp8q_policy_loss_workspace(8, 1000) - 1), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_F32, fp8q_policy_loss_workspace(8, 1000)), FP8Q_OK, 1);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_F32, 1 << 20, at<void>(2)), FP8Q_ERR_ALIGN, 0);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_BF16, 1 << 20, at<void>(2)), FP8Q_OK, 1);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_BF16, 1 << 20, nullptr), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_BF16, 1 << 20, at<void>(), 999), FP8Q_ERR_INVAL, 0);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_BF16, 1 << 20, at<void>(), WIDE), FP8Q_ERR_UNSUPPORTED, 0);
  EXPECT(loss(&b, 8, 1000, 1000, FP8Q_BF16, 1 << 20, at<void>(), 1000, at<void>(8)), FP8Q_ERR_ALIGN, 0);
  const double bad_temperatures[] = {0.0, -1.0, (double)NAN, (double)INFINITY, 1e-60, 1e60, 3.5e-39};
  for (double t : bad_temperatures) {
    b = batch();
    b.temperature = t;
    EXPECT(loss(&b), FP8Q_ERR_INVAL, 0);
  }
  b = batch();
  b.clip_low = 1.3;
  EXPECT(loss(&b), FP8Q_ERR_INVAL, 0);
  b.clip = at<fp8q_clip_result>();
  EXPECT(loss(&b), FP8Q_OK, 1);
  b.clip = at<fp8q_clip_result>(4);
  EXPECT(loss(&b), FP8Q_ERR_ALIGN, 0);
  b = batch();
  b.beta = NAN;
  EXPECT(loss(&b), FP8Q_ERR_INVAL, 0);
  b = batch();
  b.adv = nullptr;
  EXPECT(loss(&b), FP8Q_ERR_INVAL, 0);
  b = batch();
  b.w_tis = at<float>(2);
  EXPECT(loss(&b), FP8Q_ERR_ALIGN, 0);
  EXPECT(fp8q_policy_loss_workspace(BIG, 10), -1, 0);
  EXPECT(fp8q_policy_loss_workspace(10, 0), -1, 0);
  EXPECT(fp8q_token_logprobs(at<void>(), FP8Q_BF16, 8, 1000, 1000, at<int64_t>(), 1.0, at<float>(), at<float>(),
                             at<void>(), 1 << 20, nullptr), FP8Q_OK, 1);
  EXPECT(fp8q_token_logprobs(at<void>(), FP8Q_BF16, 8, 1000, 1000, at<int64_t>(4), 1.0, at<float>(), at<float>(),
                             at<void>(), 1 << 20, nullptr), FP8Q_ERR_ALIGN, 0);
  EXPECT(fp8q_token_logprobs(at<void>(1), FP8Q_BF16, 8, 1000, 1000, at<int64_t>(), 1.0, at<float>(), at<float>(),
                             at<void>(), 1 << 20, nullptr), FP8Q_ERR_ALIGN, 0);
  EXPECT(fp8q_token_logprobs(nullptr, FP8Q_BF16, 8, 1000, 1000, at<int64_t>(), 1.0, at<float>(), at<float>(),
                             at<void>(), 1 << 20, nullptr), FP8Q_ERR_INVAL, 0);
  printf("%d failures\n", failures);
  return failures != 0;
}
