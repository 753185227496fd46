// The binding's per-call work in native code: checks, output allocation, the
// current stream and the C-ABI call.  In Python these took 9-11 us a call,
// more than the kernels of a decode step or of a small layer (128 x 256 x 256,
// quantize X, quantize W, GEMM: 50 us a pass, 28 of them kernels).
//
// Every function takes exactly the calls it can prove ordinary (torch.Tensor
// or Parameter objects of the expected dtype, shape, strides and device, plain
// ints) and returns None for any other, without having done anything: the
// Python code in __init__.py then makes the call or raises the error that
// names what is wrong.  It returns the outputs, or the fp8q_status of a call
// the library refused, as an int.  The GIL is released around the library
// call, as ctypes does.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/EmptyTensor.h>
#include <ATen/core/Tensor.h>
#include <ATen/hip/impl/HIPCachingAllocatorMasqueradingAsCUDA.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <ATen/ops/empty.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/hip/HIPFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cxxabi.h>

#include <cstring>

#include "fp8q.h"

namespace {

// the library's entry points, from the loaded libfp8q.so (see bind)
struct Api {
  decltype(&fp8q_scales_count) scales_count;
  decltype(&fp8q_quantize) quantize;
  decltype(&fp8q_quantize_dual) quantize_dual;
  decltype(&fp8q_gemm_formats) gemm_formats;
  decltype(&fp8q_gemm_grouped) gemm_grouped;
  decltype(&fp8q_gemm_pow2) gemm_pow2;
  decltype(&fp8q_gemm_quantized) gemm_quantized;
  decltype(&fp8q_gemm_splitk_workspace) splitk_workspace;
  decltype(&fp8q_gemm_splitk) gemm_splitk;
  decltype(&fp8q_calibrate_clip_workspace) clip_workspace;
  decltype(&fp8q_calibrate_clip) calibrate_clip;
  decltype(&fp8q_rmsnorm) rmsnorm;
  decltype(&fp8q_rmsnorm_quantize) rmsnorm_quantize;
  decltype(&fp8q_rmsnorm_backward_workspace) norm_workspace;
  decltype(&fp8q_rmsnorm_backward) rmsnorm_backward;
  decltype(&fp8q_gemm_gated) gemm_gated;
  decltype(&fp8q_gemm_gated_workspace) gated_workspace;
  decltype(&fp8q_gemm_gated_quantized) gemm_gated_quantized;
  decltype(&fp8q_gated_backward) gated_backward;
  decltype(&fp8q_requantize_transposed) requantize_transposed;
  decltype(&fp8q_policy_loss_workspace) loss_workspace;
  decltype(&fp8q_token_logprobs) token_logprobs;
  decltype(&fp8q_policy_loss) policy_loss;
  decltype(&fp8q_quantize_mx4) quantize_mx4;
  decltype(&fp8q_dequantize_mx4) dequantize_mx4;
  decltype(&fp8q_gemm_mx4) gemm_mx4;
  decltype(&fp8q_embedding) embedding;
  decltype(&fp8q_embedding_backward_workspace) embedding_workspace;
  decltype(&fp8q_embedding_backward) embedding_backward;
  decltype(&fp8q_top_logprobs_workspace) top_workspace;
  decltype(&fp8q_top_logprobs) top_logprobs;
};
constexpr Py_ssize_t kApiSize = sizeof(Api) / sizeof(void*);

// Not an ordinary call: left to the Python code.
struct NotOrdinary {};
[[noreturn]] void leave() { throw NotOrdinary{}; }

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) leave();
  return THPVariable_Unpack(o);
}

int64_t integer(PyObject* o) {
  if (!PyLong_CheckExact(o)) leave();
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) leave();
  return v;
}

double real(PyObject* o) {
  if (!PyFloat_CheckExact(o)) leave();
  return PyFloat_AS_DOUBLE(o);
}

// t is a row-major 2-D tensor of the dtype on the GPU
const at::Tensor& matrix(PyObject* o, at::ScalarType dtype) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != dtype || t.dim() != 2 || t.stride(1) != 1) leave();
  return t;
}

// Whether nothing but the allocator takes part in at::empty: no dispatch mode or
// transform, no profiler or other observer of calls, no fill of new memory.
bool plain_allocation() {
  const at::Context& c = at::globalContext();
  return (c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() &&
         !at::hasCallbacks() && !(c.deterministicAlgorithms() && c.deterministicFillUninitializedMemory());
}

// at::empty.  On the current GPU from the caching allocator directly where that is
// all at::empty would do: a call makes up to five tensors, and the way through the
// dispatcher is half of each.
at::Tensor fresh(c10::IntArrayRef sizes, at::ScalarType dtype, c10::Device device) {
  if (device.type() == c10::DeviceType::CUDA && device.index() == c10::hip::current_device() && plain_allocation())
    return at::detail::empty_generic(sizes, c10::hip::HIPCachingAllocatorMasqueradingAsCUDA::get(),
                                     c10::DispatchKeySet(c10::DispatchKey::CUDA), dtype, std::nullopt);
  return at::empty(sizes, at::TensorOptions().dtype(dtype).device(device));
}

// the same with that shape and device, or a new one for None
at::Tensor matrix_or_new(PyObject* o, at::ScalarType dtype, int64_t rows, int64_t cols, c10::Device device) {
  if (o == Py_None) return fresh({rows, cols}, dtype, device);
  const at::Tensor& t = matrix(o, dtype);
  if (t.size(0) != rows || t.size(1) != cols || t.device() != device) leave();
  return t;
}

// t is a contiguous tensor of the dtype on the device, of n elements or more
const at::Tensor& vector(PyObject* o, at::ScalarType dtype, int64_t n, c10::Device device) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != dtype || !t.is_contiguous() ||
      t.device() != device || t.numel() < n)
    leave();
  return t;
}

at::Tensor vector_or_new(PyObject* o, at::ScalarType dtype, int64_t n, c10::Device device) {
  if (o == Py_None) return fresh({n}, dtype, device);
  return vector(o, dtype, n, device);
}

ihipStream_t* stream_of(const at::Tensor& t) {
  return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(t.device().index()).stream();
}

// The caller's object, or a new one for an output made here.
PyObject* give(PyObject* given, const at::Tensor& t) {
  if (given == Py_None) return THPVariable_Wrap(t);
  Py_INCREF(given);
  return given;
}

PyObject* pack(std::initializer_list<PyObject*> items) {
  PyObject* r = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  bool ok = r != nullptr;
  for (PyObject* o : items) {
    ok = ok && o;
    if (r) PyTuple_SET_ITEM(r, i++, o);
    else Py_XDECREF(o);
  }
  if (!ok) Py_CLEAR(r);
  return r;
}

// f() with the GIL released; f throws nothing.  Taken back by a call and not
// by a destructor: in a daemon thread that returns while the interpreter shuts
// down, PyEval_RestoreThread ends the thread by unwinding its stack, which a
// destructor (noexcept) would turn into an abort of the process.
template <typename F>
auto unlocked(F&& f) {
  PyThreadState* const s = PyEval_SaveThread();
  const auto r = f();
  PyEval_RestoreThread(s);
  return r;
}

Api* api_of(PyObject* module) { return static_cast<Api*>(PyModule_GetState(module)); }

// f(api, args), with everything it throws turned into "not an ordinary call"
// (the Python code then meets the same condition and reports it), but for the
// unwinding of a thread that ends (see unlocked), which must go on.
template <Py_ssize_t N, typename F>
PyObject* guarded(PyObject* module, PyObject* const* args, Py_ssize_t n, F&& f) {
  const Api* api = api_of(module);
  if (n == N && api->quantize) {
    try {
      return f(*api, args);
    } catch (abi::__forced_unwind&) {
      throw;
    } catch (...) {
      PyErr_Clear();
    }
  }
  Py_RETURN_NONE;
}

// quantize(x, granularity, flags, codes, scales) -> (codes, scales)
PyObject* py_quantize(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<5>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor& x = matrix(a[0], at::kBFloat16);
    const auto g = (fp8q_granularity)integer(a[1]);
    const unsigned flags = (unsigned)integer(a[2]);
    const int64_t rows = x.size(0), cols = x.size(1);
    const int64_t ns = api.scales_count(rows, cols, g, flags & FP8Q_OUT_TRANSPOSED);
    if (ns < 0) leave();
    const bool t = flags & FP8Q_OUT_TRANSPOSED;
    const at::Tensor codes = matrix_or_new(a[3], at::kByte, t ? cols : rows, t ? rows : cols, x.device());
    const at::Tensor scales = vector_or_new(a[4], at::kFloat, ns, x.device());
    const void* xp = x.const_data_ptr();
    uint8_t* cp = codes.mutable_data_ptr<uint8_t>();
    float* sp = scales.mutable_data_ptr<float>();
    ihipStream_t* s = stream_of(x);
    const fp8q_status st = unlocked([&] {
      return api.quantize(xp, rows, cols, x.stride(0), g, flags, cp, codes.stride(0), sp, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[3], codes), give(a[4], scales)});
  });
}

// quantize_dual(x, flags, codes_r, scales_r, codes_t, scales_t) -> the four
PyObject* py_quantize_dual(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<6>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor& x = matrix(a[0], at::kBFloat16);
    const unsigned flags = (unsigned)integer(a[1]);
    const int64_t rows = x.size(0), cols = x.size(1);
    const int64_t nr = api.scales_count(rows, cols, FP8Q_BLOCK_1x128, 0);
    const int64_t nt = api.scales_count(rows, cols, FP8Q_BLOCK_128x1, FP8Q_OUT_TRANSPOSED);
    if (nr < 0 || nt < 0) leave();
    const at::Tensor cr = matrix_or_new(a[2], at::kByte, rows, cols, x.device());
    const at::Tensor sr = vector_or_new(a[3], at::kFloat, nr, x.device());
    const at::Tensor ct = matrix_or_new(a[4], at::kByte, cols, rows, x.device());
    const at::Tensor sct = vector_or_new(a[5], at::kFloat, nt, x.device());
    const void* xp = x.const_data_ptr();
    uint8_t *crp = cr.mutable_data_ptr<uint8_t>(), *ctp = ct.mutable_data_ptr<uint8_t>();
    float *srp = sr.mutable_data_ptr<float>(), *stp = sct.mutable_data_ptr<float>();
    ihipStream_t* s = stream_of(x);
    const fp8q_status st = unlocked([&] {
      return api.quantize_dual(xp, rows, cols, x.stride(0), flags, crp, cr.stride(0), srp, ctp, ct.stride(0), stp, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[2], cr), give(a[3], sr), give(a[4], ct), give(a[5], sct)});
  });
}

// The operands shared by the GEMM entry points: a, sa, ga, b, sb, gb.
struct Operands {
  int64_t M, N, K, lda, ldb;
  fp8q_granularity ga, gb;
  const uint8_t *a, *b;
  const float *sa, *sb;
  c10::Device device;
  ihipStream_t* stream;
};

void operand(const Api& api, PyObject* oc, PyObject* os, fp8q_granularity g, c10::Device device, const at::Tensor*& c,
             const uint8_t*& cp, const float*& sp) {
  c = &matrix(oc, at::kByte);
  if (c->device() != device) leave();
  const int64_t ns = api.scales_count(c->size(0), c->size(1), g, 0);
  if (ns < 0) leave();
  cp = c->const_data_ptr<uint8_t>();
  sp = vector(os, at::kFloat, ns, device).const_data_ptr<float>();
}

Operands operands(const Api& api, PyObject* oa, PyObject* osa, fp8q_granularity ga, PyObject* ob, PyObject* osb,
                  fp8q_granularity gb) {
  const at::Tensor *a, *b;
  Operands p{0, 0, 0, 0, 0, ga, gb, nullptr, nullptr, nullptr, nullptr, tensor(oa).device(), nullptr};
  operand(api, oa, osa, ga, p.device, a, p.a, p.sa);
  operand(api, ob, osb, gb, p.device, b, p.b, p.sb);
  p.M = a->size(0);
  p.N = b->size(0);
  p.K = a->size(1);
  if (b->size(1) != p.K) leave();
  p.lda = a->stride(0);
  p.ldb = b->stride(0);
  p.stream = stream_of(*a);
  return p;
}

Operands operands(const Api& api, PyObject* const* a) {
  return operands(api, a[0], a[1], (fp8q_granularity)integer(a[2]), a[3], a[4], (fp8q_granularity)integer(a[5]));
}

// gemm(a, sa, ga, b, sb, gb, formats, out), gemm_pow2(a, .., gb, out) -> out
template <bool POW2>
PyObject* py_gemm(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<POW2 ? 7 : 8>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Operands p = operands(api, a);
    PyObject* const given = a[POW2 ? 6 : 7];
    const unsigned formats = POW2 ? 0u : (unsigned)integer(a[6]);
    const at::Tensor out = matrix_or_new(given, at::kBFloat16, p.M, p.N, p.device);
    void* cp = out.mutable_data_ptr();
    const fp8q_status st = unlocked([&] {
      return POW2 ? api.gemm_pow2(p.a, p.sa, p.ga, p.lda, p.b, p.sb, p.gb, p.ldb, p.M, p.N, p.K, cp, out.stride(0),
                                p.stream)
                : api.gemm_formats(p.a, p.sa, p.ga, p.lda, p.b, p.sb, p.gb, p.ldb, p.M, p.N, p.K, formats, cp,
                                   out.stride(0), p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return give(given, out);
  });
}

// gemm_splitk(a, sa, ga, b, sb, gb, out, workspace) -> out
PyObject* py_gemm_splitk(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<8>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Operands p = operands(api, a);
    const int64_t need = api.splitk_workspace(p.M, p.N, p.K);
    if (need < 0) leave();
    const at::Tensor& ws = vector(a[7], at::kByte, need, p.device);
    const at::Tensor out = matrix_or_new(a[6], at::kBFloat16, p.M, p.N, p.device);
    void *cp = out.mutable_data_ptr(), *wp = ws.mutable_data_ptr();
    const int64_t bytes = ws.numel();
    const fp8q_status st = unlocked([&] {
      return api.gemm_splitk(p.a, p.sa, p.ga, p.lda, p.b, p.sb, p.gb, p.ldb, p.M, p.N, p.K, cp, out.stride(0), wp, bytes,
                           p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return give(a[6], out);
  });
}

// gemm_quantized(a, sa, ga, b, sb, gb, codes, scales) -> (codes, scales)
PyObject* py_gemm_quantized(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<8>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Operands p = operands(api, a);
    const int64_t ns = api.scales_count(p.M, p.N, FP8Q_BLOCK_1x128, 0);
    if (ns < 0) leave();
    const at::Tensor codes = matrix_or_new(a[6], at::kByte, p.M, p.N, p.device);
    const at::Tensor scales = vector_or_new(a[7], at::kFloat, ns, p.device);
    uint8_t* cp = codes.mutable_data_ptr<uint8_t>();
    float* sp = scales.mutable_data_ptr<float>();
    const fp8q_status st = unlocked([&] {
      return api.gemm_quantized(p.a, p.sa, p.ga, p.lda, p.b, p.sb, p.gb, p.ldb, p.M, p.N, p.K, cp, codes.stride(0), sp,
                              p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[6], codes), give(a[7], scales)});
  });
}

// gemm_grouped([(a, sa, b, sb), ..], ga, gb, outs) -> outs (a list; the
// caller's object when given)
PyObject* py_gemm_grouped(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<4>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    if (!PyList_CheckExact(a[0])) leave();
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    const bool given = a[3] != Py_None;
    if (count < 1 || count > FP8Q_MAX_GROUP || (given && (!PyList_CheckExact(a[3]) || PyList_GET_SIZE(a[3]) != count)))
      leave();
    const auto ga = (fp8q_granularity)integer(a[1]), gb = (fp8q_granularity)integer(a[2]);
    fp8q_gemm_problem probs[FP8Q_MAX_GROUP];
    at::Tensor outs[FP8Q_MAX_GROUP];
    int64_t K = 0;
    c10::Device device(c10::DeviceType::CPU);
    ihipStream_t* stream = nullptr;
    for (Py_ssize_t i = 0; i < count; ++i) {
      PyObject* t = PyList_GET_ITEM(a[0], i);
      if (!PyTuple_CheckExact(t) || PyTuple_GET_SIZE(t) != 4) leave();
      const Operands p = operands(api, PyTuple_GET_ITEM(t, 0), PyTuple_GET_ITEM(t, 1), ga, PyTuple_GET_ITEM(t, 2),
                                  PyTuple_GET_ITEM(t, 3), gb);
      if (i == 0) {
        K = p.K;
        device = p.device;
        stream = p.stream;
      } else if (p.K != K || p.device != device) {
        leave();
      }
      outs[i] = matrix_or_new(given ? PyList_GET_ITEM(a[3], i) : Py_None, at::kBFloat16, p.M, p.N, device);
      probs[i] = fp8q_gemm_problem{p.a, p.sa, p.lda, p.b, p.sb, p.ldb, outs[i].mutable_data_ptr(), outs[i].stride(0), p.M, p.N};
    }
    const fp8q_status st = unlocked([&] {
      return api.gemm_grouped(probs, (int)count, ga, gb, K, stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    if (given) {
      Py_INCREF(a[3]);
      return a[3];
    }
    PyObject* list = PyList_New(count);
    for (Py_ssize_t i = 0; list && i < count; ++i) {
      PyObject* o = THPVariable_Wrap(outs[i]);
      if (!o) Py_CLEAR(list);
      else PyList_SET_ITEM(list, i, o);
    }
    return list;
  });
}

// calibrate_clip(adv, w_tis, pi_sampler, r_bf16, r_fp8, l_old, h_old, address
// of an fp8q_clip_config, workspace, result, read) -> the result's bytes with
// read (the result itself when reading it failed), else True
PyObject* py_calibrate_clip(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<11>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const float* in[5];
    const at::Tensor& adv = tensor(a[0]);
    const int64_t tokens = adv.numel();
    for (int i = 0; i < 5; ++i) {
      const at::Tensor& t = vector(a[i], at::kFloat, tokens, adv.device());
      if (t.numel() != tokens) leave();
      in[i] = t.const_data_ptr<float>();
    }
    const double l_old = real(a[5]), h_old = real(a[6]);
    const auto* config = reinterpret_cast<const fp8q_clip_config*>((uintptr_t)integer(a[7]));
    const int64_t need = api.clip_workspace(tokens);
    if (need < 0) leave();
    const at::Tensor ws = vector_or_new(a[8], at::kByte, need, adv.device());
    constexpr int64_t kResult = sizeof(fp8q_clip_result);
    const at::Tensor result = vector_or_new(a[9], at::kByte, kResult, adv.device());
    void* wp = ws.mutable_data_ptr();
    auto* rp = static_cast<fp8q_clip_result*>(result.mutable_data_ptr());
    const int64_t bytes = ws.numel();
    ihipStream_t* s = stream_of(adv);
    if (a[10] != Py_True && a[10] != Py_False) leave();
    const fp8q_status st = unlocked([&] {
      return api.calibrate_clip(in[0], in[1], in[2], in[3], in[4], tokens, l_old, h_old, config, wp, bytes, rp, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    if (a[10] == Py_False) Py_RETURN_TRUE;
    at::Tensor host;
    const bool read = unlocked([&] {  // the copy waits for the kernels
      try {
        host = result.reshape({-1}).slice(0, 0, kResult).cpu();
        return true;
      } catch (...) {
        return false;
      }
    });
    if (!read) return give(a[9], result);  // the Python code reads it again and reports why
    return PyBytes_FromStringAndSize(static_cast<const char*>(host.const_data_ptr()), kResult);
  });
}

// The norm's weight, [cols] in bf16 or fp32, and its flag.
const void* norm_weight(PyObject* o, int64_t cols, c10::Device device, unsigned& flag) {
  const at::Tensor& w = tensor(o);
  flag = w.scalar_type() == at::kFloat ? FP8Q_WEIGHT_F32 : 0u;
  if (w.dim() != 1 || w.size(0) != cols) leave();
  return vector(o, flag ? at::kFloat : at::kBFloat16, cols, device).const_data_ptr();
}

// What both norms are given but for their output, and h and rstd.
struct Norm {
  const void *x, *residual = nullptr, *weight;
  int64_t rows, cols, ldx, ldr = 0, ldh = 0;
  unsigned flag;
  void* h = nullptr;
  float* rstd;
  at::Tensor ht, rt;
  PyObject* given_h;
  c10::Device device;
  ihipStream_t* stream;
  Norm(PyObject* ox, PyObject* ow, PyObject* ores, PyObject* oh, PyObject* orstd) : device(tensor(ox).device()) {
    const at::Tensor& t = matrix(ox, at::kBFloat16);
    x = t.const_data_ptr();
    rows = t.size(0);
    cols = t.size(1);
    ldx = t.stride(0);
    stream = stream_of(t);
    weight = norm_weight(ow, cols, device, flag);
    rt = vector_or_new(orstd, at::kFloat, rows, device);
    rstd = rt.mutable_data_ptr<float>();
    given_h = oh;
    if (ores == Py_None) {
      if (oh != Py_None) leave();
      given_h = ox;  // h is x itself
      return;
    }
    const at::Tensor& r = matrix(ores, at::kBFloat16);
    if (r.size(0) != rows || r.size(1) != cols || r.device() != device) leave();
    residual = r.const_data_ptr();
    ldr = r.stride(0);
    ht = matrix_or_new(oh, at::kBFloat16, rows, cols, device);
    h = ht.mutable_data_ptr();
    ldh = ht.stride(0);
  }
};

// rmsnorm(x, weight, eps, residual, out, h, rstd) -> (out, h, rstd)
PyObject* py_rmsnorm(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<7>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Norm p(a[0], a[1], a[3], a[5], a[6]);
    const float eps = (float)real(a[2]);
    const at::Tensor y = matrix_or_new(a[4], at::kBFloat16, p.rows, p.cols, p.device);
    void* yp = y.mutable_data_ptr();
    const fp8q_status st = unlocked([&] {
      return api.rmsnorm(p.x, p.ldx, p.residual, p.ldr, p.weight, p.flag, p.rows, p.cols, eps, p.h, p.ldh, p.rstd, yp,
                         y.stride(0), p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[4], y), give(p.given_h, p.ht), give(a[6], p.rt)});
  });
}

// rmsnorm_quantize(x, weight, eps, granularity, flags, residual, codes,
// scales, h, rstd) -> (codes, scales, h, rstd)
PyObject* py_rmsnorm_quantize(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<10>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Norm p(a[0], a[1], a[5], a[8], a[9]);
    const float eps = (float)real(a[2]);
    const auto g = (fp8q_granularity)integer(a[3]);
    const unsigned flags = (unsigned)integer(a[4]) | p.flag;
    const int64_t ns = api.scales_count(p.rows, p.cols, g, 0);
    if (ns < 0) leave();
    const at::Tensor codes = matrix_or_new(a[6], at::kByte, p.rows, p.cols, p.device);
    const at::Tensor scales = vector_or_new(a[7], at::kFloat, ns, p.device);
    uint8_t* cp = codes.mutable_data_ptr<uint8_t>();
    float* sp = scales.mutable_data_ptr<float>();
    const fp8q_status st = unlocked([&] {
      return api.rmsnorm_quantize(p.x, p.ldx, p.residual, p.ldr, p.weight, flags, p.rows, p.cols, eps, p.h, p.ldh,
                                  p.rstd, g, cp, codes.stride(0), sp, p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[6], codes), give(a[7], scales), give(p.given_h, p.ht), give(a[9], p.rt)});
  });
}

// rmsnorm_backward(dy, h, rstd, weight, dres, dx, dweight, workspace) -> (dx,
// dweight)
PyObject* py_rmsnorm_backward(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<8>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor &dy = matrix(a[0], at::kBFloat16), &h = matrix(a[1], at::kBFloat16);
    const int64_t rows = dy.size(0), cols = dy.size(1);
    const c10::Device device = dy.device();
    if (h.size(0) != rows || h.size(1) != cols || h.device() != device) leave();
    const float* rstd = vector(a[2], at::kFloat, rows, device).const_data_ptr<float>();
    unsigned flag;
    const void* w = norm_weight(a[3], cols, device, flag);
    const void* dres = nullptr;
    int64_t ldres = 0;
    if (a[4] != Py_None) {
      const at::Tensor& r = matrix(a[4], at::kBFloat16);
      if (r.size(0) != rows || r.size(1) != cols || r.device() != device) leave();
      dres = r.const_data_ptr();
      ldres = r.stride(0);
    }
    const int64_t need = api.norm_workspace(rows, cols);
    if (need < 0) leave();
    const at::Tensor dx = matrix_or_new(a[5], at::kBFloat16, rows, cols, device);
    const at::Tensor dw = vector_or_new(a[6], at::kFloat, cols, device);
    const at::Tensor ws = vector_or_new(a[7], at::kByte, need, device);
    const void *dyp = dy.const_data_ptr(), *hp = h.const_data_ptr();
    void *dxp = dx.mutable_data_ptr(), *wp = ws.mutable_data_ptr();
    float* dwp = dw.mutable_data_ptr<float>();
    const int64_t bytes = ws.numel();
    ihipStream_t* s = stream_of(dy);
    const fp8q_status st = unlocked([&] {
      return api.rmsnorm_backward(dyp, dy.stride(0), hp, h.stride(0), rstd, w, flag, dres, ldres, rows, cols, dxp,
                                  dx.stride(0), dwp, wp, bytes, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[5], dx), give(a[6], dw)});
  });
}

bool truth(PyObject* o) {
  if (o != Py_True && o != Py_False) leave();
  return o == Py_True;
}

// gemm_gated(a, sa, b, sb, save, out, pre) -> (out, pre) and
// gemm_gated_quantized(a, sa, b, sb, save, codes, scales, pre, workspace) ->
// (codes, scales, pre)
template <bool QOUT>
PyObject* py_gemm_gated(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<QOUT ? 9 : 7>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Operands p = operands(api, a[0], a[1], FP8Q_BLOCK_1x128, a[2], a[3], FP8Q_BLOCK_128x128);
    PyObject* const given_pre = a[QOUT ? 7 : 6];
    if (p.N % 2) leave();
    const int64_t F = p.N / 2;
    at::Tensor pre;
    void* pp = nullptr;
    int64_t ldp = 0;
    if (truth(a[4]) || given_pre != Py_None) {
      pre = matrix_or_new(given_pre, at::kBFloat16, p.M, p.N, p.device);
      pp = pre.mutable_data_ptr();
      ldp = pre.stride(0);
    }
    auto kept = [&]() -> PyObject* {
      if (pp) return give(given_pre, pre);
      Py_RETURN_NONE;
    };
    if (QOUT) {
      const int64_t ns = api.scales_count(p.M, F, FP8Q_BLOCK_1x128, 0);
      if (ns < 0) leave();
      const at::Tensor codes = matrix_or_new(a[5], at::kByte, p.M, F, p.device);
      const at::Tensor scales = vector_or_new(a[6], at::kFloat, ns, p.device);
      uint8_t* cp = codes.mutable_data_ptr<uint8_t>();
      float* sp = scales.mutable_data_ptr<float>();
      const int64_t need = api.gated_workspace(p.M, F, p.K);
      if (need < 0) leave();
      at::Tensor ws;
      void* wp = nullptr;
      int64_t bytes = 0;
      if (need > 0) {
        ws = vector_or_new(a[8], at::kByte, need, p.device);
        wp = ws.mutable_data_ptr();
        bytes = ws.numel();
      }
      const fp8q_status st = unlocked([&] {
        return api.gemm_gated_quantized(p.a, p.sa, p.lda, p.b, p.sb, p.ldb, p.M, F, p.K, pp, ldp, cp, codes.stride(0),
                                        sp, wp, bytes, p.stream);
      });
      if (st != FP8Q_OK) return PyLong_FromLong(st);
      return pack({give(a[5], codes), give(a[6], scales), kept()});
    }
    const at::Tensor out = matrix_or_new(a[5], at::kBFloat16, p.M, F, p.device);
    void* op = out.mutable_data_ptr();
    const fp8q_status st = unlocked([&] {
      return api.gemm_gated(p.a, p.sa, p.lda, p.b, p.sb, p.ldb, p.M, F, p.K, op, out.stride(0), pp, ldp, p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[5], out), kept()});
  });
}

// gated_backward(dh, pre, flags, codes_r, scales_r, codes_t, scales_t) -> the
// four
PyObject* py_gated_backward(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<7>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor &dh = matrix(a[0], at::kBFloat16), &pre = matrix(a[1], at::kBFloat16);
    const unsigned flags = (unsigned)integer(a[2]);
    const int64_t M = dh.size(0), F = dh.size(1), Mp = (M + 127) / 128 * 128;
    const c10::Device device = dh.device();
    if (pre.size(0) != M || pre.size(1) != 2 * F || pre.device() != device) leave();
    const at::Tensor cr = matrix_or_new(a[3], at::kByte, M, 2 * F, device);
    const at::Tensor sr = vector_or_new(a[4], at::kFloat, M * (2 * F / 128), device);
    const at::Tensor ct = matrix_or_new(a[5], at::kByte, 2 * F, Mp, device);
    const at::Tensor sct = vector_or_new(a[6], at::kFloat, Mp / 128 * 2 * F, device);
    const void *dhp = dh.const_data_ptr(), *pp = pre.const_data_ptr();
    uint8_t *crp = cr.mutable_data_ptr<uint8_t>(), *ctp = ct.mutable_data_ptr<uint8_t>();
    float *srp = sr.mutable_data_ptr<float>(), *stp = sct.mutable_data_ptr<float>();
    ihipStream_t* s = stream_of(dh);
    const fp8q_status st = unlocked([&] {
      return api.gated_backward(dhp, dh.stride(0), pp, pre.stride(0), M, F, flags, crp, cr.stride(0), srp, ctp,
                                ct.stride(0), stp, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[3], cr), give(a[4], sr), give(a[5], ct), give(a[6], sct)});
  });
}

// requantize_transposed(codes, scales, flags, codes_t, scales_t) -> (codes_t,
// scales_t)
PyObject* py_requantize_transposed(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<5>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor& codes = matrix(a[0], at::kByte);
    const unsigned flags = (unsigned)integer(a[2]);
    const int64_t rows = codes.size(0), cols = codes.size(1), Rp = (rows + 127) / 128 * 128;
    const c10::Device device = codes.device();
    const int64_t ns = api.scales_count(rows, cols, FP8Q_BLOCK_1x128, 0);
    if (ns < 0) leave();
    const float* sp = vector(a[1], at::kFloat, ns, device).const_data_ptr<float>();
    const at::Tensor ct = matrix_or_new(a[3], at::kByte, cols, Rp, device);
    const at::Tensor sct = vector_or_new(a[4], at::kFloat, Rp / 128 * cols, device);
    const uint8_t* cp = codes.const_data_ptr<uint8_t>();
    uint8_t* ctp = ct.mutable_data_ptr<uint8_t>();
    float* stp = sct.mutable_data_ptr<float>();
    ihipStream_t* s = stream_of(codes);
    const fp8q_status st = unlocked([&] {
      return api.requantize_transposed(cp, codes.stride(0), sp, rows, cols, flags, ctp, ct.stride(0), stp, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[3], ct), give(a[4], sct)});
  });
}

// Logits, tokens and workspace of the two calls on them.
struct Logits {
  const void* x;
  fp8q_dtype dtype;
  int64_t T, V, ld, bytes;
  const int64_t* tokens;
  at::Tensor ws;
  void* wp;
  c10::Device device;
  ihipStream_t* stream;
  Logits(const Api& api, PyObject* ox, PyObject* ot, PyObject* ow) : device(tensor(ox).device()) {
    dtype = tensor(ox).scalar_type() == at::kFloat ? FP8Q_F32 : FP8Q_BF16;
    const at::Tensor& t = matrix(ox, type());
    x = t.const_data_ptr();
    T = t.size(0);
    V = t.size(1);
    ld = t.stride(0);
    tokens = vector(ot, at::kLong, T, device).const_data_ptr<int64_t>();
    const int64_t need = api.loss_workspace(T, V);
    if (need < 0) leave();
    ws = vector_or_new(ow, at::kByte, need, device);
    wp = ws.mutable_data_ptr();
    bytes = ws.numel();
    stream = stream_of(t);
  }
  at::ScalarType type() const { return dtype == FP8Q_F32 ? at::kFloat : at::kBFloat16; }
};

// token_logprobs(logits, tokens, temperature, logp, entropy, workspace) ->
// (logp, entropy)
PyObject* py_token_logprobs(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<6>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Logits p(api, a[0], a[1], a[5]);
    const double temperature = real(a[2]);
    const at::Tensor logp = vector_or_new(a[3], at::kFloat, p.T, p.device);
    const at::Tensor entropy = vector_or_new(a[4], at::kFloat, p.T, p.device);
    float *lp = logp.mutable_data_ptr<float>(), *ep = entropy.mutable_data_ptr<float>();
    const fp8q_status st = unlocked([&] {
      return api.token_logprobs(p.x, p.dtype, p.T, p.V, p.ld, p.tokens, temperature, lp, ep, p.wp, p.bytes, p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[3], logp), give(a[4], entropy)});
  });
}

// policy_loss(logits, tokens, logp_old, adv, weight, clip_low, clip_high,
// beta, logp_ref, w_tis, temperature, clip, loss, dlogits, logp, entropy,
// workspace) -> (loss, dlogits, logp, entropy)
PyObject* py_policy_loss(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<17>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const Logits p(api, a[0], a[1], a[16]);
    auto tokenwise = [&](PyObject* o) { return vector(o, at::kFloat, p.T, p.device).const_data_ptr<float>(); };
    fp8q_policy_batch b{};
    b.tokens = p.tokens;
    b.logp_old = tokenwise(a[2]);
    b.adv = tokenwise(a[3]);
    b.weight = tokenwise(a[4]);
    if (a[8] != Py_None) b.logp_ref = tokenwise(a[8]);
    if (a[9] != Py_None) b.w_tis = tokenwise(a[9]);
    b.clip_low = real(a[5]);
    b.clip_high = real(a[6]);
    b.beta = real(a[7]);
    b.temperature = real(a[10]);
    if (a[11] != Py_None)
      b.clip = static_cast<const fp8q_clip_result*>(
          vector(a[11], at::kByte, sizeof(fp8q_clip_result), p.device).const_data_ptr());
    const at::Tensor loss = vector_or_new(a[12], at::kFloat, 1, p.device);
    const at::Tensor dlogits = matrix_or_new(a[13], p.type(), p.T, p.V, p.device);
    const at::Tensor logp = vector_or_new(a[14], at::kFloat, p.T, p.device);
    const at::Tensor entropy = vector_or_new(a[15], at::kFloat, p.T, p.device);
    float *lossp = loss.mutable_data_ptr<float>(), *lp = logp.mutable_data_ptr<float>();
    float* ep = entropy.mutable_data_ptr<float>();
    void* dp = dlogits.mutable_data_ptr();
    const fp8q_status st = unlocked([&] {
      return api.policy_loss(p.x, p.dtype, p.T, p.V, p.ld, &b, lossp, dp, dlogits.stride(0), lp, ep, p.wp, p.bytes,
                             p.stream);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[12], loss), give(a[13], dlogits), give(a[14], logp), give(a[15], entropy)});
  });
}

// Bytes of MXFP4 codes that a row of cols elements takes, and of its scales.
int64_t mx4_row_bytes(int64_t cols) { return (cols + 255) / 256 * 128; }

// MXFP4 operands: codes [rows, K / 2] with the scales of their rows.
struct Mx4 {
  const uint8_t *codes, *scales;
  int64_t rows, K, ld;
  Mx4(PyObject* oc, PyObject* os, c10::Device device) {
    const at::Tensor& c = matrix(oc, at::kByte);
    if (c.device() != device || c.size(1) % 128) leave();
    rows = c.size(0);
    K = c.size(1) * 2;
    ld = c.stride(0);
    codes = c.const_data_ptr<uint8_t>();
    scales = vector(os, at::kByte, rows * (K / 32), device).const_data_ptr<uint8_t>();
  }
};

// quantize_mx4(x, codes, scales) -> (codes, scales)
PyObject* py_quantize_mx4(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<3>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor& x = matrix(a[0], at::kBFloat16);
    const int64_t rows = x.size(0), cols = x.size(1), bytes = mx4_row_bytes(cols);
    const at::Tensor codes = matrix_or_new(a[1], at::kByte, rows, bytes, x.device());
    const at::Tensor scales = vector_or_new(a[2], at::kByte, rows * (bytes / 16), x.device());
    const void* xp = x.const_data_ptr();
    uint8_t *cp = codes.mutable_data_ptr<uint8_t>(), *sp = scales.mutable_data_ptr<uint8_t>();
    ihipStream_t* s = stream_of(x);
    const fp8q_status st = unlocked([&] {
      return api.quantize_mx4(xp, rows, cols, x.stride(0), cp, codes.stride(0), sp, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[1], codes), give(a[2], scales)});
  });
}

// dequantize_mx4(codes, scales, cols, out) -> out
PyObject* py_dequantize_mx4(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<4>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const c10::Device device = tensor(a[0]).device();
    const Mx4 q(a[0], a[1], device);
    const int64_t cols = integer(a[2]);
    if (cols < 1 || cols > q.K) leave();
    const at::Tensor out = matrix_or_new(a[3], at::kBFloat16, q.rows, cols, device);
    void* yp = out.mutable_data_ptr();
    ihipStream_t* s = stream_of(out);
    const fp8q_status st = unlocked([&] {
      return api.dequantize_mx4(q.codes, q.ld, q.scales, q.rows, cols, yp, out.stride(0), s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return give(a[3], out);
  });
}

// gemm_mx4(a, sa, b, sb, out) -> out
PyObject* py_gemm_mx4(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<5>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const c10::Device device = tensor(a[0]).device();
    const Mx4 p(a[0], a[1], device), q(a[2], a[3], device);
    if (p.K != q.K || (a[4] == Py_None && q.rows % 4)) leave();
    const at::Tensor out = matrix_or_new(a[4], at::kBFloat16, p.rows, q.rows, device);
    void* cp = out.mutable_data_ptr();
    ihipStream_t* s = stream_of(out);
    const fp8q_status st = unlocked([&] {
      return api.gemm_mx4(p.codes, p.scales, p.ld, q.codes, q.scales, q.ld, p.rows, q.rows, p.K, cp, out.stride(0), s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return give(a[4], out);
  });
}

// embedding(weight, tokens, scale, out) -> out
PyObject* py_embedding(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<4>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const fp8q_dtype dtype = tensor(a[0]).scalar_type() == at::kFloat ? FP8Q_F32 : FP8Q_BF16;
    const at::Tensor& w = matrix(a[0], dtype == FP8Q_F32 ? at::kFloat : at::kBFloat16);
    const at::Tensor& tokens = vector(a[1], at::kLong, 0, w.device());
    if (tokens.dim() != 1) leave();
    const double scale = real(a[2]);
    const int64_t T = tokens.size(0), V = w.size(0), C = w.size(1);
    const at::Tensor out = matrix_or_new(a[3], at::kBFloat16, T, C, w.device());
    const void* wp = w.const_data_ptr();
    const int64_t* tp = tokens.const_data_ptr<int64_t>();
    void* yp = out.mutable_data_ptr();
    ihipStream_t* s = stream_of(w);
    const fp8q_status st = unlocked([&] {
      return api.embedding(wp, dtype, V, C, w.stride(0), tp, T, scale, yp, out.stride(0), s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return give(a[3], out);
  });
}

// embedding_backward(dy, tokens, vocab, scale, f32, dweight, accumulate, workspace) -> dweight
PyObject* py_embedding_backward(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<8>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const at::Tensor& dy = matrix(a[0], at::kBFloat16);
    const c10::Device device = dy.device();
    const at::Tensor& tokens = vector(a[1], at::kLong, 0, device);
    const int64_t T = dy.size(0), C = dy.size(1), V = integer(a[2]);
    if (tokens.dim() != 1 || tokens.size(0) != T) leave();
    const double scale = real(a[3]);
    const bool f32 = truth(a[4]), accumulate = truth(a[6]);
    if (accumulate && a[5] == Py_None) leave();
    const int64_t need = api.embedding_workspace(T, V, C);
    if (need < 0) leave();
    const at::Tensor dw = matrix_or_new(a[5], f32 ? at::kFloat : at::kBFloat16, V, C, device);
    const at::Tensor ws = vector_or_new(a[7], at::kByte, need, device);
    const void* dyp = dy.const_data_ptr();
    const int64_t* tp = tokens.const_data_ptr<int64_t>();
    void *dwp = dw.mutable_data_ptr(), *wp = ws.mutable_data_ptr();
    const int64_t bytes = ws.numel();
    ihipStream_t* s = stream_of(dy);
    const fp8q_status st = unlocked([&] {
      return api.embedding_backward(dyp, dy.stride(0), tp, T, V, C, scale, accumulate ? FP8Q_ACCUMULATE : 0u, dwp,
                                    f32 ? FP8Q_F32 : FP8Q_BF16, dw.stride(0), wp, bytes, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return give(a[5], dw);
  });
}

// top_logprobs(logits, tokens, k, temperature, logp, entropy, ids, top, workspace) -> (logp,
// entropy, ids, top)
PyObject* py_top_logprobs(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  return guarded<9>(m, a, n, [](const Api& api, PyObject* const* a) -> PyObject* {
    const fp8q_dtype dtype = tensor(a[0]).scalar_type() == at::kFloat ? FP8Q_F32 : FP8Q_BF16;
    const at::Tensor& x = matrix(a[0], dtype == FP8Q_F32 ? at::kFloat : at::kBFloat16);
    const c10::Device device = x.device();
    const int64_t T = x.size(0), V = x.size(1), k = integer(a[2]);
    const int64_t* tokens = vector(a[1], at::kLong, T, device).const_data_ptr<int64_t>();
    const double temperature = real(a[3]);
    const int64_t need = api.top_workspace(T, V, k);
    if (need < 0) leave();
    const at::Tensor logp = vector_or_new(a[4], at::kFloat, T, device);
    const at::Tensor entropy = vector_or_new(a[5], at::kFloat, T, device);
    auto contiguous = [&](PyObject* o, at::ScalarType type) {
      const at::Tensor t = matrix_or_new(o, type, T, k, device);
      if (!t.is_contiguous()) leave();
      return t;
    };
    const at::Tensor ids = contiguous(a[6], at::kLong), top = contiguous(a[7], at::kFloat);
    at::Tensor ws;
    void* wp = nullptr;
    int64_t bytes = 0;
    if (need > 0) {
      ws = vector_or_new(a[8], at::kByte, need, device);
      wp = ws.mutable_data_ptr();
      bytes = ws.numel();
    }
    const void* xp = x.const_data_ptr();
    float *lp = logp.mutable_data_ptr<float>(), *ep = entropy.mutable_data_ptr<float>();
    int64_t* ip = ids.mutable_data_ptr<int64_t>();
    float* kp = top.mutable_data_ptr<float>();
    ihipStream_t* s = stream_of(x);
    const fp8q_status st = unlocked([&] {
      return api.top_logprobs(xp, dtype, T, V, x.stride(0), tokens, k, temperature, lp, ep, ip, kp, wp, bytes, s);
    });
    if (st != FP8Q_OK) return PyLong_FromLong(st);
    return pack({give(a[4], logp), give(a[5], entropy), give(a[6], ids), give(a[7], top)});
  });
}

// bind((address, ..)): the entry points of Api, in its order
PyObject* py_bind(PyObject* m, PyObject* addresses) {
  if (!PyTuple_CheckExact(addresses) || PyTuple_GET_SIZE(addresses) != kApiSize) {
    PyErr_SetString(PyExc_ValueError, "bind: a tuple of the entry points' addresses");
    return nullptr;
  }
  void* p[kApiSize];
  for (Py_ssize_t i = 0; i < kApiSize; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: a null address");
      return nullptr;
    }
  }
  std::memcpy(static_cast<void*>(api_of(m)), p, sizeof p);
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", py_bind, METH_O, nullptr},
    {"quantize", FAST(py_quantize), nullptr},
    {"quantize_dual", FAST(py_quantize_dual), nullptr},
    {"gemm", FAST(py_gemm<false>), nullptr},
    {"gemm_pow2", FAST(py_gemm<true>), nullptr},
    {"gemm_splitk", FAST(py_gemm_splitk), nullptr},
    {"gemm_quantized", FAST(py_gemm_quantized), nullptr},
    {"gemm_grouped", FAST(py_gemm_grouped), nullptr},
    {"calibrate_clip", FAST(py_calibrate_clip), nullptr},
    {"rmsnorm", FAST(py_rmsnorm), nullptr},
    {"rmsnorm_quantize", FAST(py_rmsnorm_quantize), nullptr},
    {"rmsnorm_backward", FAST(py_rmsnorm_backward), nullptr},
    {"gemm_gated", FAST(py_gemm_gated<false>), nullptr},
    {"gemm_gated_quantized", FAST(py_gemm_gated<true>), nullptr},
    {"gated_backward", FAST(py_gated_backward), nullptr},
    {"requantize_transposed", FAST(py_requantize_transposed), nullptr},
    {"token_logprobs", FAST(py_token_logprobs), nullptr},
    {"policy_loss", FAST(py_policy_loss), nullptr},
    {"quantize_mx4", FAST(py_quantize_mx4), nullptr},
    {"dequantize_mx4", FAST(py_dequantize_mx4), nullptr},
    {"gemm_mx4", FAST(py_gemm_mx4), nullptr},
    {"embedding", FAST(py_embedding), nullptr},
    {"embedding_backward", FAST(py_embedding_backward), nullptr},
    {"top_logprobs", FAST(py_top_logprobs), nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, sizeof(Api), methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
  PyObject* m = PyModule_Create(&module);
  if (m) std::memset(PyModule_GetState(m), 0, sizeof(Api));
  return m;
}
