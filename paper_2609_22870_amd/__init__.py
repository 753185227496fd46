"""fp8q: FP8 scaled quantization (paper Sec. 2.2, Eq. 3) and the scaled FP8
GEMM of the FP8 linear layer, as hand-written HIP kernels for MI355X (gfx950).

This module is a thin binding over the C-ABI of ``libfp8q.so`` (declared in
``include/fp8q.h``): it only marshals arguments.  PyTorch is used for device
memory and the current HIP stream; every step of the computation runs in the
library's kernels.  There is no fallback: if the library is missing, every
call raises.

Each wrapper first hands its arguments to the function of ``_native.so``
(csrc/binding.cpp) that checks, allocates and calls the C-ABI in native code;
that takes ordinary calls and returns None for any other, which the Python
code below then makes, or refuses with the error that says why.
"""
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfp8q.so")

# fp8q_granularity
TENSOR, ROW, COL, BLOCK_1x128, BLOCK_128x1, BLOCK_128x128 = range(6)
OUT_TRANSPOSED = 1
POW2_SCALE = 2
ACCUMULATE = 32               # embedding_backward flag: dweight is added to
MAX_TOP = 64                  # alternatives of top_logprobs, at most
E5M2 = 4                      # quantize flag: E5M2 codes (F_max = 57344)
WEIGHT_F32 = 16               # norm flag: its weight is fp32
A_E5M2, B_E5M2 = 1, 2         # gemm_formats operand formats
_STATUS = {0: "FP8Q_OK", -1: "FP8Q_ERR_INVAL", -2: "FP8Q_ERR_UNSUPPORTED",
           -3: "FP8Q_ERR_ALIGN", -4: "FP8Q_ERR_HIP"}
# the entry points of include/fp8q.h
EXPORTS = ("fp8q_scales_count", "fp8q_quantize", "fp8q_quantize_dual",
           "fp8q_gemm", "fp8q_gemm_grouped", "fp8q_gemm_formats", "fp8q_gemm_pow2", "fp8q_gemm_quantized",
           "fp8q_gemm_splitk_workspace", "fp8q_gemm_splitk",
           "fp8q_calibrate_clip_workspace", "fp8q_calibrate_clip", "fp8q_calibrate_clip_noalloc",
           "fp8q_cast_f32",
           "fp8q_cast_f32_e5m2", "fp8q_rmsnorm", "fp8q_rmsnorm_quantize", "fp8q_rmsnorm_backward_workspace",
           "fp8q_rmsnorm_backward", "fp8q_gemm_gated", "fp8q_gemm_gated_workspace", "fp8q_gemm_gated_quantized",
           "fp8q_gated_backward",
           "fp8q_requantize_transposed", "fp8q_policy_loss_workspace", "fp8q_token_logprobs", "fp8q_policy_loss",
           "fp8q_quantize_mx4", "fp8q_dequantize_mx4", "fp8q_gemm_mx4", "fp8q_embedding",
           "fp8q_embedding_backward_workspace", "fp8q_embedding_backward", "fp8q_top_logprobs_workspace",
           "fp8q_top_logprobs", "fp8q_status_string")


MAX_GROUP = 8


class GemmProblem(ctypes.Structure):
    """fp8q_gemm_problem of include/fp8q.h."""
    _fields_ = [("A", ctypes.c_void_p), ("sA", ctypes.c_void_p), ("lda", ctypes.c_int64),
                ("B", ctypes.c_void_p), ("sB", ctypes.c_void_p), ("ldb", ctypes.c_int64),
                ("C", ctypes.c_void_p), ("ldc", ctypes.c_int64),
                ("M", ctypes.c_int64), ("N", ctypes.c_int64)]


class ClipConfig(ctypes.Structure):
    """fp8q_clip_config (include/fp8q.h)."""
    _fields_ = [(n, ctypes.c_double) for n in ("c_low_ref", "c_high_ref", "l_min", "l_max",
                                                "h_min", "h_max", "step", "delta_l", "delta_h")]


class ClipResult(ctypes.Structure):
    """fp8q_clip_result (include/fp8q.h)."""
    _fields_ = ([(n, ctypes.c_double) for n in ("l_new", "h_new", "l_star", "h_star", "alpha_low",
                                                 "rho_bf16", "rho_fp8")]
                + [("n_neg", ctypes.c_int64), ("n_pos", ctypes.c_int64),
                   ("l_updated", ctypes.c_int32), ("h_updated", ctypes.c_int32)])


class PolicyBatch(ctypes.Structure):
    """fp8q_policy_batch (include/fp8q.h)."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("tokens", "logp_old", "adv", "weight", "w_tis", "logp_ref", "clip")]
                + [(n, ctypes.c_double) for n in ("clip_low", "clip_high", "beta", "temperature")])


_CLIP_FIELDS = tuple(n for n, _ in ClipResult._fields_)
_CLIP_STRUCT = struct.Struct("=7d2q2i")


# Sec. 4 settings, with the GRPO experiments' reference bounds (Sec. 5.1).
PAPER_CLIP_CONFIG = dict(c_low_ref=0.8, c_high_ref=1.24, l_min=0.5, l_max=0.9, h_min=1.2,
                         h_max=2.0, step=0.02, delta_l=0.05, delta_h=0.1)


class Fp8qError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s: %s" % (what, status_string(status)))


_lib = None
_calls = None
# the entry points of binding.cpp's Api, in its order
_NATIVE_API = ("fp8q_scales_count", "fp8q_quantize", "fp8q_quantize_dual", "fp8q_gemm_formats", "fp8q_gemm_grouped",
               "fp8q_gemm_pow2", "fp8q_gemm_quantized", "fp8q_gemm_splitk_workspace", "fp8q_gemm_splitk",
               "fp8q_calibrate_clip_workspace", "fp8q_calibrate_clip", "fp8q_rmsnorm", "fp8q_rmsnorm_quantize",
               "fp8q_rmsnorm_backward_workspace", "fp8q_rmsnorm_backward", "fp8q_gemm_gated",
               "fp8q_gemm_gated_workspace", "fp8q_gemm_gated_quantized", "fp8q_gated_backward",
               "fp8q_requantize_transposed",
               "fp8q_policy_loss_workspace", "fp8q_token_logprobs", "fp8q_policy_loss", "fp8q_quantize_mx4",
               "fp8q_dequantize_mx4", "fp8q_gemm_mx4", "fp8q_embedding", "fp8q_embedding_backward_workspace",
               "fp8q_embedding_backward", "fp8q_top_logprobs_workspace", "fp8q_top_logprobs")


def lib():
    """Load libfp8q.so (built by __graft_entry__.build()); raise if absent."""
    global _lib, _calls
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libfp8q.so is not built (%s); run "
                              "__graft_entry__.build()" % LIB_PATH)
        from . import _native as native  # ImportError when it is not built
        L = ctypes.CDLL(LIB_PATH)
        p, i64, i32, u32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint
        L.fp8q_scales_count.argtypes = [i64, i64, i32, u32]
        L.fp8q_scales_count.restype = i64
        L.fp8q_quantize.argtypes = [p, i64, i64, i64, i32, u32, p, i64, p, p]
        L.fp8q_quantize.restype = i32
        L.fp8q_quantize_dual.argtypes = [p, i64, i64, i64, u32, p, i64, p, p, i64, p, p]
        L.fp8q_quantize_dual.restype = i32
        L.fp8q_gemm.argtypes = [p, p, i32, i64, p, p, i32, i64, i64, i64, i64,
                                p, i64, p]
        L.fp8q_gemm.restype = i32
        L.fp8q_gemm_grouped.argtypes = [ctypes.POINTER(GemmProblem), i32, i32, i32, i64, p]
        L.fp8q_gemm_grouped.restype = i32
        L.fp8q_gemm_formats.argtypes = [p, p, i32, i64, p, p, i32, i64, i64, i64, i64, u32, p, i64, p]
        L.fp8q_gemm_formats.restype = i32
        L.fp8q_gemm_pow2.argtypes = [p, p, i32, i64, p, p, i32, i64, i64, i64, i64, p, i64, p]
        L.fp8q_gemm_pow2.restype = i32
        L.fp8q_gemm_quantized.argtypes = [p, p, i32, i64, p, p, i32, i64, i64,
                                          i64, i64, p, i64, p, p]
        L.fp8q_gemm_quantized.restype = i32
        L.fp8q_gemm_splitk_workspace.argtypes = [i64, i64, i64]
        L.fp8q_gemm_splitk_workspace.restype = i64
        L.fp8q_gemm_splitk.argtypes = [p, p, i32, i64, p, p, i32, i64, i64, i64, i64,
                                       p, i64, p, i64, p]
        L.fp8q_gemm_splitk.restype = i32
        L.fp8q_calibrate_clip_workspace.argtypes = [i64]
        L.fp8q_calibrate_clip_workspace.restype = i64
        d = ctypes.c_double
        L.fp8q_calibrate_clip.argtypes = [p, p, p, p, p, i64, d, d, ctypes.POINTER(ClipConfig),
                                          p, i64, p, p]
        L.fp8q_calibrate_clip.restype = i32
        L.fp8q_calibrate_clip_noalloc.argtypes = [p, p, p, p, p, i64, d, d, ctypes.POINTER(ClipConfig), p, p]
        L.fp8q_calibrate_clip_noalloc.restype = i32
        L.fp8q_cast_f32.argtypes = [p, i64, ctypes.c_float, p, p]
        L.fp8q_cast_f32_e5m2.argtypes = [p, i64, ctypes.c_float, p, p]
        L.fp8q_cast_f32_e5m2.restype = i32
        L.fp8q_cast_f32.restype = i32
        f32 = ctypes.c_float
        L.fp8q_rmsnorm.argtypes = [p, i64, p, i64, p, u32, i64, i64, f32, p, i64, p, p, i64, p]
        L.fp8q_rmsnorm.restype = i32
        L.fp8q_rmsnorm_quantize.argtypes = [p, i64, p, i64, p, u32, i64, i64, f32, p, i64, p, i32, p, i64, p, p]
        L.fp8q_rmsnorm_quantize.restype = i32
        L.fp8q_rmsnorm_backward_workspace.argtypes = [i64, i64]
        L.fp8q_rmsnorm_backward_workspace.restype = i64
        L.fp8q_rmsnorm_backward.argtypes = [p, i64, p, i64, p, p, u32, p, i64, i64, i64, p, i64, p, p, i64, p]
        L.fp8q_rmsnorm_backward.restype = i32
        L.fp8q_gemm_gated.argtypes = [p, p, i64, p, p, i64, i64, i64, i64, p, i64, p, i64, p]
        L.fp8q_gemm_gated.restype = i32
        L.fp8q_gemm_gated_workspace.argtypes = [i64, i64, i64]
        L.fp8q_gemm_gated_workspace.restype = i64
        L.fp8q_gemm_gated_quantized.argtypes = [p, p, i64, p, p, i64, i64, i64, i64, p, i64, p, i64, p, p, i64, p]
        L.fp8q_gemm_gated_quantized.restype = i32
        L.fp8q_gated_backward.argtypes = [p, i64, p, i64, i64, i64, u32, p, i64, p, p, i64, p, p]
        L.fp8q_gated_backward.restype = i32
        L.fp8q_requantize_transposed.argtypes = [p, i64, p, i64, i64, u32, p, i64, p, p]
        L.fp8q_requantize_transposed.restype = i32
        L.fp8q_policy_loss_workspace.argtypes = [i64, i64]
        L.fp8q_policy_loss_workspace.restype = i64
        L.fp8q_token_logprobs.argtypes = [p, i32, i64, i64, i64, p, d, p, p, p, i64, p]
        L.fp8q_token_logprobs.restype = i32
        L.fp8q_policy_loss.argtypes = [p, i32, i64, i64, i64, ctypes.POINTER(PolicyBatch), p, p, i64, p, p, p, i64, p]
        L.fp8q_policy_loss.restype = i32
        L.fp8q_quantize_mx4.argtypes = [p, i64, i64, i64, p, i64, p, p]
        L.fp8q_quantize_mx4.restype = i32
        L.fp8q_dequantize_mx4.argtypes = [p, i64, p, i64, i64, p, i64, p]
        L.fp8q_dequantize_mx4.restype = i32
        L.fp8q_gemm_mx4.argtypes = [p, p, i64, p, p, i64, i64, i64, i64, p, i64, p]
        L.fp8q_gemm_mx4.restype = i32
        L.fp8q_embedding.argtypes = [p, i32, i64, i64, i64, p, i64, d, p, i64, p]
        L.fp8q_embedding.restype = i32
        L.fp8q_embedding_backward_workspace.argtypes = [i64, i64, i64]
        L.fp8q_embedding_backward_workspace.restype = i64
        L.fp8q_embedding_backward.argtypes = [p, i64, p, i64, i64, i64, d, u32, p, i32, i64, p, i64, p]
        L.fp8q_embedding_backward.restype = i32
        L.fp8q_top_logprobs_workspace.argtypes = [i64, i64, i64]
        L.fp8q_top_logprobs_workspace.restype = i64
        L.fp8q_top_logprobs.argtypes = [p, i32, i64, i64, i64, p, i64, d, p, p, p, p, p, i64, p]
        L.fp8q_top_logprobs.restype = i32
        L.fp8q_status_string.argtypes = [i32]
        L.fp8q_status_string.restype = ctypes.c_char_p
        native.bind(tuple(ctypes.cast(getattr(L, n), p).value for n in _NATIVE_API))
        _calls = native
        _lib = L
    return _lib


def status_string(status):
    try:
        return lib().fp8q_status_string(status).decode()
    except ImportError:
        return _STATUS.get(status, str(status))


def _fast():
    """The native entry points (the library loaded)."""
    if _lib is None:
        lib()
    return _calls


def _check(status, what):
    if status != 0:
        raise Fp8qError(status, what)


def _done(r, what):
    """The native call's outputs, or its status as an error."""
    if type(r) is int:
        raise Fp8qError(r, what)
    return r


def _stream(t):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def _ld(t):
    """Leading dimension of a row-major 2-D tensor (unit column stride)."""
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("expected a row-major 2-D tensor")
    return t.stride(0)


def _matrix(t, dtype, what, shape=None, device=None):
    """t as a row-major 2-D CUDA tensor of dtype (and of shape / on device
    when given): the kernels read and write exactly that region, so a
    tensor of another shape would be read or written past its end."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda or t.dim() != 2:
        raise ValueError("%s must be a 2-D %s CUDA tensor" % (what, dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, not %s" % (what, tuple(shape), tuple(t.shape)))
    if device is not None and t.device != device:
        raise ValueError("%s must be on %s" % (what, device))
    _ld(t)
    return t


def _vector(t, dtype, n, what, device):
    """t as a contiguous CUDA tensor of dtype with at least n elements."""
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda or not t.is_contiguous()
            or t.device != device):
        raise ValueError("%s must be a contiguous %s tensor on %s" % (what, dtype, device))
    if t.numel() < n:
        raise ValueError("%s holds %d elements, %d needed" % (what, t.numel(), n))
    return t


def _operands(a, sa, ga, b, sb, gb):
    """The checks shared by the GEMM entry points: FP8 codes a [M, K] and b
    [N, K] on one device, and scale arrays holding at least the counts
    their granularities give for those shapes; returns M, N, K."""
    _matrix(a, torch.uint8, "a")
    _matrix(b, torch.uint8, "b", device=a.device)
    M, K = a.shape
    N, K2 = b.shape
    if K != K2:
        raise ValueError("contraction sizes differ")
    _vector(sa, torch.float32, max(scales_count(M, K, ga), 0), "sa", a.device)
    _vector(sb, torch.float32, max(scales_count(N, K, gb), 0), "sb", a.device)
    return M, N, K


def scales_count(rows, cols, granularity, transposed=False):
    n = lib().fp8q_scales_count(rows, cols, granularity, OUT_TRANSPOSED if transposed else 0)
    if n < 0:
        raise ValueError("invalid quantization shape or granularity")
    return n


def quantize(x, granularity, transposed=False, codes=None, scales=None, pow2=False, e5m2=False):
    """Eq. 3 per scaling unit on a bf16 CUDA tensor x[rows, cols].

    Returns (codes, scales): codes uint8 (OCP E4M3 bytes) [rows, cols], or
    [cols, rows] when `transposed`; scales fp32 1-D in the layout of
    include/fp8q.h.  pow2: power-of-two scales (FP8Q_POW2_SCALE); e5m2:
    E5M2 codes (FP8Q_E5M2).
    """
    flags = (OUT_TRANSPOSED if transposed else 0) | (POW2_SCALE if pow2 else 0) | (E5M2 if e5m2 else 0)
    r = _fast().quantize(x, granularity, flags, codes, scales)
    if r is not None:
        return _done(r, "fp8q_quantize")
    _matrix(x, torch.bfloat16, "x")
    rows, cols = x.shape
    oshape = (cols, rows) if transposed else (rows, cols)
    n = scales_count(rows, cols, granularity, transposed)
    if codes is None:
        codes = torch.empty(oshape, dtype=torch.uint8, device=x.device)
    _matrix(codes, torch.uint8, "codes", oshape, x.device)
    if scales is None:
        scales = torch.empty(n, dtype=torch.float32, device=x.device)
    _vector(scales, torch.float32, n, "scales", x.device)
    st = lib().fp8q_quantize(x.data_ptr(), rows, cols, _ld(x), granularity, flags,
                             codes.data_ptr(), _ld(codes), scales.data_ptr(),
                             _stream(x))
    _check(st, "fp8q_quantize")
    return codes, scales


def quantize_dual(x, codes_r=None, scales_r=None, codes_t=None, scales_t=None, pow2=False, e5m2=False):
    """Both backward-pass layouts of a bf16 CUDA tensor x[rows, cols] from
    one read: (codes_r, scales_r) = quantize(x, BLOCK_1x128) and
    (codes_t, scales_t) = quantize(x, BLOCK_128x1, transposed=True), with
    the same pow2 / e5m2 options."""
    flags = (POW2_SCALE if pow2 else 0) | (E5M2 if e5m2 else 0)
    r = _fast().quantize_dual(x, flags, codes_r, scales_r, codes_t, scales_t)
    if r is not None:
        return _done(r, "fp8q_quantize_dual")
    _matrix(x, torch.bfloat16, "x")
    rows, cols = x.shape
    nr, nt = scales_count(rows, cols, BLOCK_1x128), scales_count(rows, cols, BLOCK_128x1, True)
    if codes_r is None:
        codes_r = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    if scales_r is None:
        scales_r = torch.empty(nr, dtype=torch.float32, device=x.device)
    if codes_t is None:
        codes_t = torch.empty((cols, rows), dtype=torch.uint8, device=x.device)
    if scales_t is None:
        scales_t = torch.empty(nt, dtype=torch.float32, device=x.device)
    _matrix(codes_r, torch.uint8, "codes_r", (rows, cols), x.device)
    _matrix(codes_t, torch.uint8, "codes_t", (cols, rows), x.device)
    _vector(scales_r, torch.float32, nr, "scales_r", x.device)
    _vector(scales_t, torch.float32, nt, "scales_t", x.device)
    st = lib().fp8q_quantize_dual(x.data_ptr(), rows, cols, _ld(x), flags,
                                  codes_r.data_ptr(), _ld(codes_r),
                                  scales_r.data_ptr(), codes_t.data_ptr(),
                                  _ld(codes_t), scales_t.data_ptr(), _stream(x))
    _check(st, "fp8q_quantize_dual")
    return codes_r, scales_r, codes_t, scales_t


def gemm(a, sa, ga, b, sb, gb, out=None):
    """C[M, N] = dequant(a)[M, K] @ dequant(b)[N, K]^T in bf16.

    a, b: uint8 E4M3 codes, K contiguous; sa, sb: fp32 scales for the
    granularities ga, gb (pairs listed in include/fp8q.h).
    """
    r = _fast().gemm(a, sa, ga, b, sb, gb, 0, out)
    if r is not None:
        return _done(r, "fp8q_gemm")
    M, N, K = _operands(a, sa, ga, b, sb, gb)
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    _matrix(out, torch.bfloat16, "out", (M, N), a.device)
    st = lib().fp8q_gemm(a.data_ptr(), sa.data_ptr(), ga, _ld(a),
                         b.data_ptr(), sb.data_ptr(), gb, _ld(b), M, N, K,
                         out.data_ptr(), _ld(out), _stream(a))
    _check(st, "fp8q_gemm")
    return out


def gemm_splitk_workspace(M, N, K):
    """Bytes of workspace gemm_splitk needs for an M x N x K problem (0 when
    it does not split K)."""
    need = lib().fp8q_gemm_splitk_workspace(M, N, K)
    if need < 0:
        raise ValueError("invalid GEMM size")
    return need


def gemm_splitk(a, sa, ga, b, sb, gb, out=None, workspace=None):
    """gemm for skinny problems with each output tile's K blocks split over
    several workgroups (fp8q_gemm_splitk).  workspace: a uint8 CUDA tensor
    of at least gemm_splitk_workspace(M, N, K) bytes, zero-filled before its
    first use (a new zero-filled one when None); calls sharing it must be
    ordered (one stream)."""
    r = _fast().gemm_splitk(a, sa, ga, b, sb, gb, out, workspace)
    if r is not None:
        return _done(r, "fp8q_gemm_splitk")
    M, N, K = _operands(a, sa, ga, b, sb, gb)
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    _matrix(out, torch.bfloat16, "out", (M, N), a.device)
    need = gemm_splitk_workspace(M, N, K)
    if workspace is None:
        workspace = torch.zeros(max(need, 16), dtype=torch.uint8, device=a.device)
    _vector(workspace, torch.uint8, need, "workspace", a.device)
    st = lib().fp8q_gemm_splitk(a.data_ptr(), sa.data_ptr(), ga, _ld(a),
                                b.data_ptr(), sb.data_ptr(), gb, _ld(b), M, N, K,
                                out.data_ptr(), _ld(out), workspace.data_ptr(),
                                workspace.numel(), _stream(a))
    _check(st, "fp8q_gemm_splitk")
    return out


def gemm_grouped(problems, ga, gb, outs=None):
    """Several gemm() problems in one launch (fp8q_gemm_grouped).

    problems: list of (a, sa, b, sb) with one K and the granularities ga,
    gb for all (the a's may be the same tensor); returns the bf16 outputs
    (or fills `outs`)."""
    r = _fast().gemm_grouped(problems, ga, gb, outs)
    if r is not None:
        return _done(r, "fp8q_gemm_grouped")
    if not 1 <= len(problems) <= MAX_GROUP:
        raise ValueError("1 .. %d problems" % MAX_GROUP)
    K = problems[0][0].shape[1]
    dev = problems[0][0].device
    for a, sa, b, sb in problems:
        _operands(a, sa, ga, b, sb, gb)
        if a.shape[1] != K or a.device != dev:
            raise ValueError("every problem must have the same K and device")
    if outs is None:
        outs = [torch.empty((a.shape[0], b.shape[0]), dtype=torch.bfloat16, device=a.device)
                for a, _, b, _ in problems]
    if len(outs) != len(problems):
        raise ValueError("one output per problem")
    arr = (GemmProblem * len(problems))()
    for i, ((a, sa, b, sb), c) in enumerate(zip(problems, outs)):
        _matrix(c, torch.bfloat16, "outs[%d]" % i, (a.shape[0], b.shape[0]), dev)
        arr[i] = GemmProblem(a.data_ptr(), sa.data_ptr(), _ld(a), b.data_ptr(), sb.data_ptr(), _ld(b),
                             c.data_ptr(), _ld(c), a.shape[0], b.shape[0])
    st = lib().fp8q_gemm_grouped(arr, len(problems), ga, gb, K, _stream(problems[0][0]))
    _check(st, "fp8q_gemm_grouped")
    return outs


def gemm_formats(a, sa, ga, b, sb, gb, formats, out=None):
    """gemm() with E5M2 codes for A (formats & A_E5M2) and/or B (formats &
    B_E5M2): the backward pairs (1x128, 128x128) and (1x128, 1x128)."""
    r = _fast().gemm(a, sa, ga, b, sb, gb, formats, out)
    if r is not None:
        return _done(r, "fp8q_gemm_formats")
    M, N, K = _operands(a, sa, ga, b, sb, gb)
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    _matrix(out, torch.bfloat16, "out", (M, N), a.device)
    st = lib().fp8q_gemm_formats(a.data_ptr(), sa.data_ptr(), ga, _ld(a),
                                 b.data_ptr(), sb.data_ptr(), gb, _ld(b), M, N, K,
                                 formats, out.data_ptr(), _ld(out), _stream(a))
    _check(st, "fp8q_gemm_formats")
    return out


def gemm_pow2(a, sa, ga, b, sb, gb, out=None):
    """gemm() for operands quantized with power-of-two scales (pow2=True):
    the block scales enter the matrix instruction as exponents."""
    r = _fast().gemm_pow2(a, sa, ga, b, sb, gb, out)
    if r is not None:
        return _done(r, "fp8q_gemm_pow2")
    M, N, K = _operands(a, sa, ga, b, sb, gb)
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    _matrix(out, torch.bfloat16, "out", (M, N), a.device)
    st = lib().fp8q_gemm_pow2(a.data_ptr(), sa.data_ptr(), ga, _ld(a),
                              b.data_ptr(), sb.data_ptr(), gb, _ld(b), M, N, K,
                              out.data_ptr(), _ld(out), _stream(a))
    _check(st, "fp8q_gemm_pow2")
    return out


def gemm_quantized(a, sa, ga, b, sb, gb, codes=None, scales=None):
    """The GEMM of gemm() with its bf16 output quantized per 1x128 block
    (the next layer's activation operand), in one kernel.  Returns (codes
    uint8 [M, N], scales fp32 in the 1x128 layout), exactly
    quantize(gemm(a, sa, ga, b, sb, gb), BLOCK_1x128)."""
    r = _fast().gemm_quantized(a, sa, ga, b, sb, gb, codes, scales)
    if r is not None:
        return _done(r, "fp8q_gemm_quantized")
    M, N, K = _operands(a, sa, ga, b, sb, gb)
    n = scales_count(M, N, BLOCK_1x128)
    if codes is None:
        codes = torch.empty((M, N), dtype=torch.uint8, device=a.device)
    if scales is None:
        scales = torch.empty(n, dtype=torch.float32, device=a.device)
    _matrix(codes, torch.uint8, "codes", (M, N), a.device)
    _vector(scales, torch.float32, n, "scales", a.device)
    st = lib().fp8q_gemm_quantized(a.data_ptr(), sa.data_ptr(), ga, _ld(a),
                                   b.data_ptr(), sb.data_ptr(), gb, _ld(b), M, N, K,
                                   codes.data_ptr(), _ld(codes), scales.data_ptr(),
                                   _stream(a))
    _check(st, "fp8q_gemm_quantized")
    return codes, scales


def calibrate_clip(adv, w_tis, pi_sampler, r_bf16, r_fp8, l_old, h_old, config=None,
                   workspace=None, result=None, read=True):
    """Calibrated Clipping (Alg. 1) on the GPU.  The five per-token inputs
    are contiguous float32 CUDA tensors of one batch; config maps the
    fields of ClipConfig (default: the paper's).  Returns the result as a
    dict (reading it back waits for the kernels); `result` may be a uint8
    CUDA tensor of ctypes.sizeof(ClipResult) bytes to write into, and with
    read=False nothing is read back (the call returns None)."""
    cfg = ClipConfig(**(config or PAPER_CLIP_CONFIG))
    r = _fast().calibrate_clip(adv, w_tis, pi_sampler, r_bf16, r_fp8, l_old, h_old, ctypes.addressof(cfg),
                               workspace, result, bool(read))
    if r is not None:
        r = _done(r, "fp8q_calibrate_clip")
        if r is True:
            return None
        if isinstance(r, torch.Tensor):
            r = r.cpu().numpy().tobytes()
        return dict(zip(_CLIP_FIELDS, _CLIP_STRUCT.unpack_from(r)))
    ts = (adv, w_tis, pi_sampler, r_bf16, r_fp8)
    n = adv.numel()
    for t in ts:
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
            raise ValueError("inputs must be contiguous float32 CUDA tensors of one length")
    need = lib().fp8q_calibrate_clip_workspace(n)
    if need < 0:
        raise ValueError("empty batch")
    if workspace is None:
        workspace = torch.empty(max(need, 8), dtype=torch.uint8, device=adv.device)
    if result is None:
        result = torch.empty(ctypes.sizeof(ClipResult), dtype=torch.uint8, device=adv.device)
    _vector(workspace, torch.uint8, need, "workspace", adv.device)
    _vector(result, torch.uint8, ctypes.sizeof(ClipResult), "result", adv.device)
    st = lib().fp8q_calibrate_clip(*(t.data_ptr() for t in ts), n, float(l_old), float(h_old),
                                   ctypes.byref(cfg), workspace.data_ptr(), workspace.numel(),
                                   result.data_ptr(), _stream(adv))
    _check(st, "fp8q_calibrate_clip")
    if not read:
        return None
    r = ClipResult.from_buffer_copy(result.cpu().numpy().tobytes())
    return {name: getattr(r, name) for name, _ in ClipResult._fields_}


def calibrate_clip_noalloc(adv, w_tis, pi_sampler, r_bf16, r_fp8, l_old, h_old, config=None,
                           result=None, read=True):
    """calibrate_clip() through fp8q_calibrate_clip_noalloc: no workspace,
    the partial sums go to the library's own device array (calls on one
    device must not overlap).  `result` and `read` as for calibrate_clip."""
    ts = (adv, w_tis, pi_sampler, r_bf16, r_fp8)
    n = adv.numel()
    for t in ts:
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
            raise ValueError("inputs must be contiguous float32 CUDA tensors of one length")
    cfg = ClipConfig(**(config or PAPER_CLIP_CONFIG))
    if result is None:
        result = torch.empty(ctypes.sizeof(ClipResult), dtype=torch.uint8, device=adv.device)
    _vector(result, torch.uint8, ctypes.sizeof(ClipResult), "result", adv.device)
    st = lib().fp8q_calibrate_clip_noalloc(*(t.data_ptr() for t in ts), n, float(l_old), float(h_old),
                                           ctypes.byref(cfg), result.data_ptr(), _stream(adv))
    _check(st, "fp8q_calibrate_clip_noalloc")
    if not read:
        return None
    r = ClipResult.from_buffer_copy(result.cpu().numpy().tobytes())
    return {name: getattr(r, name) for name, _ in ClipResult._fields_}


def cast_f32(x, scale, codes=None, e5m2=False):
    """Q_FP8(RN32(x / scale)) elementwise on an fp32 CUDA tensor (E4M3, or
    E5M2 codes)."""
    if x.dtype != torch.float32 or not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous fp32 CUDA tensor")
    if codes is None:
        codes = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    _vector(codes, torch.uint8, x.numel(), "codes", x.device)
    fn = lib().fp8q_cast_f32_e5m2 if e5m2 else lib().fp8q_cast_f32
    st = fn(x.data_ptr(), x.numel(), float(scale), codes.data_ptr(), _stream(x))
    _check(st, "fp8q_cast_f32_e5m2" if e5m2 else "fp8q_cast_f32")
    return codes


def _given(t, dtype, what, shape, device):
    """The output t checked, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    return _matrix(t, dtype, what, shape, device)


def _new_vector(t, dtype, n, what, device):
    """The vector t checked, or a new one of n elements."""
    return torch.empty(n, dtype=dtype, device=device) if t is None else _vector(t, dtype, n, what, device)


def _norm_weight(weight, cols, device):
    """The norm's weight checked, and its flag."""
    if not isinstance(weight, torch.Tensor) or weight.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("weight must be a bfloat16 or float32 tensor")
    _vector(weight, weight.dtype, cols, "weight", device)
    if weight.dim() != 1 or weight.numel() != cols:
        raise ValueError("weight must have one element per column")
    return WEIGHT_F32 if weight.dtype == torch.float32 else 0


def _norm_inputs(x, weight, residual, h, rstd):
    """The checks and outputs that both norms share: (flag, h, rstd, the C
    arguments for the residual and for h)."""
    _matrix(x, torch.bfloat16, "x")
    rows, cols = x.shape
    flag = _norm_weight(weight, cols, x.device)
    rstd = _new_vector(rstd, torch.float32, rows, "rstd", x.device)
    if residual is None:
        if h is not None:
            raise ValueError("h is x itself without a residual")
        return flag, x, rstd, (None, 0), (None, 0)
    _matrix(residual, torch.bfloat16, "residual", x.shape, x.device)
    h = _given(h, torch.bfloat16, "h", (rows, cols), x.device)
    return flag, h, rstd, (residual.data_ptr(), _ld(residual)), (h.data_ptr(), _ld(h))


def rmsnorm(x, weight, eps, residual=None, out=None, h=None, rstd=None):
    """RMS norm of a bf16 CUDA tensor x[rows, cols], or of h = bf16(x +
    residual): returns (y, h, rstd), y = h rstd weight in bf16, h the new
    residual stream (x itself without a residual; `h` may be x or residual)
    and rstd fp32 [rows], which rmsnorm_backward takes.  weight: bf16 or fp32
    [cols]."""
    r = _fast().rmsnorm(x, weight, eps, residual, out, h, rstd)
    if r is not None:
        return _done(r, "fp8q_rmsnorm")
    flag, h, rstd, res, ho = _norm_inputs(x, weight, residual, h, rstd)
    out = _given(out, torch.bfloat16, "out", tuple(x.shape), x.device)
    st = lib().fp8q_rmsnorm(x.data_ptr(), _ld(x), *res, weight.data_ptr(), flag, *x.shape, float(eps), *ho,
                            rstd.data_ptr(), out.data_ptr(), _ld(out), _stream(x))
    _check(st, "fp8q_rmsnorm")
    return out, h, rstd


def rmsnorm_quantize(x, weight, eps, granularity=BLOCK_1x128, residual=None, pow2=False, codes=None, scales=None,
                     h=None, rstd=None):
    """rmsnorm() with y in 8 bits, quantized from its fp32 values: returns
    (codes, scales, h, rstd), codes and scales as quantize() gives them for
    `granularity` (BLOCK_1x128 or ROW), a GEMM's operand."""
    flags = POW2_SCALE if pow2 else 0
    r = _fast().rmsnorm_quantize(x, weight, eps, granularity, flags, residual, codes, scales, h, rstd)
    if r is not None:
        return _done(r, "fp8q_rmsnorm_quantize")
    flag, h, rstd, res, ho = _norm_inputs(x, weight, residual, h, rstd)
    rows, cols = x.shape
    codes = _given(codes, torch.uint8, "codes", (rows, cols), x.device)
    scales = _new_vector(scales, torch.float32, scales_count(rows, cols, granularity), "scales", x.device)
    st = lib().fp8q_rmsnorm_quantize(x.data_ptr(), _ld(x), *res, weight.data_ptr(), flag | flags, rows, cols,
                                     float(eps), *ho, rstd.data_ptr(), granularity, codes.data_ptr(), _ld(codes),
                                     scales.data_ptr(), _stream(x))
    _check(st, "fp8q_rmsnorm_quantize")
    return codes, scales, h, rstd


def rmsnorm_backward(dy, h, rstd, weight, dres=None, dx=None, dweight=None, workspace=None):
    """Gradients of rmsnorm() from that of y, with h and rstd as it returned
    them and `dres` the gradient that reaches h past the norm: returns (dx,
    dweight), dx in bf16 the gradient of x and of the residual alike (`dx`
    may be dy or dres), dweight fp32 [cols].  workspace: a uint8 CUDA tensor
    of fp8q_rmsnorm_backward_workspace bytes (a new one when None)."""
    r = _fast().rmsnorm_backward(dy, h, rstd, weight, dres, dx, dweight, workspace)
    if r is not None:
        return _done(r, "fp8q_rmsnorm_backward")
    _matrix(dy, torch.bfloat16, "dy")
    rows, cols = dy.shape
    dev = dy.device
    _matrix(h, torch.bfloat16, "h", dy.shape, dev)
    _vector(rstd, torch.float32, rows, "rstd", dev)
    flag = _norm_weight(weight, cols, dev)
    if dres is not None:
        _matrix(dres, torch.bfloat16, "dres", dy.shape, dev)
    dx = _given(dx, torch.bfloat16, "dx", (rows, cols), dev)
    dweight = _new_vector(dweight, torch.float32, cols, "dweight", dev)
    need = max(lib().fp8q_rmsnorm_backward_workspace(rows, cols), 0)
    workspace = _new_vector(workspace, torch.uint8, max(need, 16), "workspace", dev)
    st = lib().fp8q_rmsnorm_backward(dy.data_ptr(), _ld(dy), h.data_ptr(), _ld(h), rstd.data_ptr(), weight.data_ptr(),
                                     flag, None if dres is None else dres.data_ptr(), 0 if dres is None else _ld(dres),
                                     rows, cols, dx.data_ptr(), _ld(dx), dweight.data_ptr(), workspace.data_ptr(),
                                     workspace.numel(), _stream(dy))
    _check(st, "fp8q_rmsnorm_backward")
    return dx, dweight


def _gated_operands(a, sa, b, sb, save, pre):
    """The checks that both gated GEMMs share: (M, F, K, pre, its C arguments)."""
    M, N, K = _operands(a, sa, BLOCK_1x128, b, sb, BLOCK_128x128)
    if N % 2:
        raise ValueError("b holds the rows of two weights")
    if save or pre is not None:
        pre = _given(pre, torch.bfloat16, "pre", (M, N), a.device)
        return M, N // 2, K, pre, (pre.data_ptr(), _ld(pre))
    return M, N // 2, K, None, (None, 0)


def gemm_gated(a, sa, b, sb, save=False, out=None, pre=None):
    """H = silu(X Wg^T) * (X Wu^T) in one kernel, for a gated feed-forward
    block on FP8 operands: a, sa the codes and 1x128 scales of X [M, K]; b, sb
    those of the two weights one below the other, [2 F, K] with 128x128
    scales.  Returns (h, pre): h bf16 [M, F]; pre the pre-activations [M, 2 F]
    (gate, then up) for gated_backward when `save` (or given), else None."""
    r = _fast().gemm_gated(a, sa, b, sb, save, out, pre)
    if r is not None:
        return _done(r, "fp8q_gemm_gated")
    M, F, K, pre, pc = _gated_operands(a, sa, b, sb, save, pre)
    out = _given(out, torch.bfloat16, "out", (M, F), a.device)
    st = lib().fp8q_gemm_gated(a.data_ptr(), sa.data_ptr(), _ld(a), b.data_ptr(), sb.data_ptr(), _ld(b), M, F, K,
                               out.data_ptr(), _ld(out), *pc, _stream(a))
    _check(st, "fp8q_gemm_gated")
    return out, pre


def gemm_gated_quantized(a, sa, b, sb, save=False, codes=None, scales=None, pre=None, workspace=None):
    """gemm_gated() with H in 8 bits, the down projection's operand: returns
    (codes, scales, pre), exactly quantize(h, BLOCK_1x128) of its h.
    workspace: a uint8 CUDA tensor of fp8q_gemm_gated_workspace bytes (a new
    one when None and the size needs one)."""
    r = _fast().gemm_gated_quantized(a, sa, b, sb, save, codes, scales, pre, workspace)
    if r is not None:
        return _done(r, "fp8q_gemm_gated_quantized")
    M, F, K, pre, pc = _gated_operands(a, sa, b, sb, save, pre)
    codes = _given(codes, torch.uint8, "codes", (M, F), a.device)
    scales = _new_vector(scales, torch.float32, scales_count(M, F, BLOCK_1x128), "scales", a.device)
    need = max(lib().fp8q_gemm_gated_workspace(M, F, K), 0)
    workspace = _new_vector(workspace, torch.uint8, need, "workspace", a.device)
    st = lib().fp8q_gemm_gated_quantized(a.data_ptr(), sa.data_ptr(), _ld(a), b.data_ptr(), sb.data_ptr(), _ld(b), M, F,
                                         K, *pc, codes.data_ptr(), _ld(codes), scales.data_ptr(),
                                         workspace.data_ptr() if need else None, workspace.numel(), _stream(a))
    _check(st, "fp8q_gemm_gated_quantized")
    return codes, scales, pre


def _padded(rows):
    """rows rounded up to whole units of 128."""
    return (rows + 127) // 128 * 128


def gated_backward(dh, pre, pow2=False, e5m2=False, codes_r=None, scales_r=None, codes_t=None, scales_t=None):
    """Gradients of gemm_gated()'s pre-activations from that of h, as the FP8
    operands of the backward GEMMs: D = [dG | dU], M x 2 F.  Returns
    (codes_r, scales_r, codes_t, scales_t): D per 1x128 unit, for dX = D W,
    and D^T per 128x1 unit, [2 F, Mp], for [dWg; dWu] = D^T X, Mp being M
    rounded up to a multiple of 128 (zeros there).  pow2, e5m2: as in
    quantize()."""
    flags = (POW2_SCALE if pow2 else 0) | (E5M2 if e5m2 else 0)
    r = _fast().gated_backward(dh, pre, flags, codes_r, scales_r, codes_t, scales_t)
    if r is not None:
        return _done(r, "fp8q_gated_backward")
    _matrix(dh, torch.bfloat16, "dh")
    M, F = dh.shape
    dev = dh.device
    _matrix(pre, torch.bfloat16, "pre", (M, 2 * F), dev)
    codes_r = _given(codes_r, torch.uint8, "codes_r", (M, 2 * F), dev)
    codes_t = _given(codes_t, torch.uint8, "codes_t", (2 * F, _padded(M)), dev)
    scales_r = _new_vector(scales_r, torch.float32, M * (2 * F // 128), "scales_r", dev)
    scales_t = _new_vector(scales_t, torch.float32, _padded(M) // 128 * 2 * F, "scales_t", dev)
    st = lib().fp8q_gated_backward(dh.data_ptr(), _ld(dh), pre.data_ptr(), _ld(pre), M, F, flags, codes_r.data_ptr(),
                                   _ld(codes_r), scales_r.data_ptr(), codes_t.data_ptr(), _ld(codes_t),
                                   scales_t.data_ptr(), _stream(dh))
    _check(st, "fp8q_gated_backward")
    return codes_r, scales_r, codes_t, scales_t


def requantize_transposed(codes, scales, pow2=False, codes_t=None, scales_t=None):
    """The weight gradient's operand from an activation kept in 8 bits: codes
    [rows, cols] (E4M3) with 1x128 scales in, (codes_t, scales_t) out, the
    transpose [cols, Rp] per 128x1 unit, Rp being rows rounded up to a
    multiple of 128 (zeros there).  pow2: power-of-two scales."""
    r = _fast().requantize_transposed(codes, scales, POW2_SCALE if pow2 else 0, codes_t, scales_t)
    if r is not None:
        return _done(r, "fp8q_requantize_transposed")
    _matrix(codes, torch.uint8, "codes")
    rows, cols = codes.shape
    dev = codes.device
    _vector(scales, torch.float32, scales_count(rows, cols, BLOCK_1x128), "scales", dev)
    codes_t = _given(codes_t, torch.uint8, "codes_t", (cols, _padded(rows)), dev)
    scales_t = _new_vector(scales_t, torch.float32, _padded(rows) // 128 * cols, "scales_t", dev)
    st = lib().fp8q_requantize_transposed(codes.data_ptr(), _ld(codes), scales.data_ptr(), rows, cols,
                                          POW2_SCALE if pow2 else 0, codes_t.data_ptr(), _ld(codes_t),
                                          scales_t.data_ptr(), _stream(codes))
    _check(st, "fp8q_requantize_transposed")
    return codes_t, scales_t


def _logits(logits, tokens, workspace):
    """The checks that the two calls on logits share: (their type's code, T, V,
    workspace)."""
    if not isinstance(logits, torch.Tensor) or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be a 2-D bfloat16 or float32 CUDA tensor")
    _matrix(logits, logits.dtype, "logits")
    T, V = logits.shape
    _vector(tokens, torch.int64, T, "tokens", logits.device)
    need = lib().fp8q_policy_loss_workspace(T, V)
    if need < 0:
        raise ValueError("invalid number of tokens or vocabulary size")
    return 1 if logits.dtype == torch.float32 else 0, T, V, _new_vector(workspace, torch.uint8, need, "workspace",
                                                                        logits.device)


def token_logprobs(logits, tokens, temperature=1.0, logp=None, entropy=None, workspace=None):
    """Log-probabilities of `tokens` (int64 [T]) under softmax(logits /
    temperature), logits bf16 or fp32 [T, V], and the rows' entropies: returns
    (logp, entropy), fp32 [T].  A token outside the vocabulary gives 0 and 0.
    workspace: a uint8 CUDA tensor of fp8q_policy_loss_workspace bytes (a new
    one when None)."""
    r = _fast().token_logprobs(logits, tokens, temperature, logp, entropy, workspace)
    if r is not None:
        return _done(r, "fp8q_token_logprobs")
    dtype, T, V, workspace = _logits(logits, tokens, workspace)
    logp = _new_vector(logp, torch.float32, T, "logp", logits.device)
    entropy = _new_vector(entropy, torch.float32, T, "entropy", logits.device)
    st = lib().fp8q_token_logprobs(logits.data_ptr(), dtype, T, V, _ld(logits), tokens.data_ptr(), float(temperature),
                                   logp.data_ptr(), entropy.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                   _stream(logits))
    _check(st, "fp8q_token_logprobs")
    return logp, entropy


def policy_loss(logits, tokens, logp_old, adv, weight, clip_low, clip_high, beta=0.0, logp_ref=None, w_tis=None,
                temperature=1.0, clip=None, loss=None, dlogits=None, logp=None, entropy=None, workspace=None):
    """The clipped policy loss with truncated importance sampling and a KL
    term, and its gradient in the logits (see fp8q_policy_loss): returns
    (loss [1], dlogits, logp, entropy).  tokens int64 [T]; logp_old, adv,
    weight (0: the token does not count) and, optionally, logp_ref and w_tis
    fp32 [T]; clip: the `result` tensor of calibrate_clip(), whose new bounds
    then replace clip_low and clip_high without a copy to the host; `dlogits`
    may be the logits."""
    r = _fast().policy_loss(logits, tokens, logp_old, adv, weight, clip_low, clip_high, beta, logp_ref, w_tis,
                            temperature, clip, loss, dlogits, logp, entropy, workspace)
    if r is not None:
        return _done(r, "fp8q_policy_loss")
    dtype, T, V, workspace = _logits(logits, tokens, workspace)
    dev = logits.device
    batch = PolicyBatch(tokens=tokens.data_ptr(), clip_low=float(clip_low), clip_high=float(clip_high),
                        beta=float(beta), temperature=float(temperature))
    for name, t in (("logp_old", logp_old), ("adv", adv), ("weight", weight), ("w_tis", w_tis), ("logp_ref", logp_ref)):
        if t is not None or name in ("logp_old", "adv", "weight"):
            setattr(batch, name, _vector(t, torch.float32, T, name, dev).data_ptr())
    if clip is not None:
        batch.clip = _vector(clip, torch.uint8, ctypes.sizeof(ClipResult), "clip", dev).data_ptr()
    loss = _new_vector(loss, torch.float32, 1, "loss", dev)
    dlogits = _given(dlogits, logits.dtype, "dlogits", (T, V), dev)
    logp = _new_vector(logp, torch.float32, T, "logp", dev)
    entropy = _new_vector(entropy, torch.float32, T, "entropy", dev)
    st = lib().fp8q_policy_loss(logits.data_ptr(), dtype, T, V, _ld(logits), ctypes.byref(batch), loss.data_ptr(),
                                dlogits.data_ptr(), _ld(dlogits), logp.data_ptr(), entropy.data_ptr(),
                                workspace.data_ptr(), workspace.numel(), _stream(logits))
    _check(st, "fp8q_policy_loss")
    return loss, dlogits, logp, entropy


def _mx4_row_bytes(cols):
    """Bytes of MXFP4 codes of a row of cols elements (its length rounded up to a multiple of 256)."""
    return (cols + 255) // 256 * 128


def _mx4(codes, scales, what, device=None):
    """MXFP4 operands checked: codes [rows, K / 2] and the scales of their rows; returns rows, K."""
    _matrix(codes, torch.uint8, what, device=device)
    rows, row_bytes = codes.shape
    if row_bytes % 128:
        raise ValueError("%s must have whole pieces of 256 codes in a row" % what)
    _vector(scales, torch.uint8, rows * (row_bytes // 16), "scales of %s" % what, codes.device)
    return rows, row_bytes * 2


def quantize_mx4(x, codes=None, scales=None):
    """MXFP4 (E2M1 codes, a power-of-two scale per 32 elements of a row) of a bf16 CUDA
    tensor x[rows, cols]: returns (codes, scales), an operand of gemm_mx4().  With P =
    cols rounded up to a multiple of 256: codes uint8 [rows, P / 2], two a byte, the first in
    the low half, zeros past cols; scales uint8 [rows * P / 32], exponent + 127, laid out
    [P / 256][rows][8] (see fp8q_quantize_mx4)."""
    r = _fast().quantize_mx4(x, codes, scales)
    if r is not None:
        return _done(r, "fp8q_quantize_mx4")
    _matrix(x, torch.bfloat16, "x")
    rows, cols = x.shape
    codes = _given(codes, torch.uint8, "codes", (rows, _mx4_row_bytes(cols)), x.device)
    scales = _new_vector(scales, torch.uint8, rows * (_mx4_row_bytes(cols) // 16), "scales", x.device)
    st = lib().fp8q_quantize_mx4(x.data_ptr(), rows, cols, _ld(x), codes.data_ptr(), _ld(codes), scales.data_ptr(),
                                 _stream(x))
    _check(st, "fp8q_quantize_mx4")
    return codes, scales


def dequantize_mx4(codes, scales, cols=None, out=None):
    """The values of MXFP4 codes as quantize_mx4() gives them, bf16 [rows, cols]: the first
    `cols` elements of each row (all of them, with the zeros that fill it up, when None)."""
    if cols is None and isinstance(codes, torch.Tensor) and codes.dim() == 2:
        cols = codes.shape[1] * 2
    r = _fast().dequantize_mx4(codes, scales, cols, out)
    if r is not None:
        return _done(r, "fp8q_dequantize_mx4")
    rows, K = _mx4(codes, scales, "codes")
    if not 1 <= cols <= K:
        raise ValueError("cols must lie in 1 .. %d" % K)
    out = _given(out, torch.bfloat16, "out", (rows, cols), codes.device)
    st = lib().fp8q_dequantize_mx4(codes.data_ptr(), _ld(codes), scales.data_ptr(), rows, cols, out.data_ptr(), _ld(out),
                                   _stream(codes))
    _check(st, "fp8q_dequantize_mx4")
    return out


def gemm_mx4(a, sa, b, sb, out=None):
    """bf16 out[M, N] = A B^T of MXFP4 operands as quantize_mx4() gives them: a, sa the codes
    [M, K / 2] and scales of the activations, b, sb those of a weight stored [N, K]; fp32
    accumulation.  Rows of out lie a multiple of 4 elements apart: a new one of another N has
    room behind each row."""
    r = _fast().gemm_mx4(a, sa, b, sb, out)
    if r is not None:
        return _done(r, "fp8q_gemm_mx4")
    M, K = _mx4(a, sa, "a")
    N, K2 = _mx4(b, sb, "b", a.device)
    if K != K2:
        raise ValueError("contraction sizes differ")
    if out is None:
        out = torch.empty((M, -(-N // 4) * 4), dtype=torch.bfloat16, device=a.device)[:, :N]
    _matrix(out, torch.bfloat16, "out", (M, N), a.device)
    st = lib().fp8q_gemm_mx4(a.data_ptr(), sa.data_ptr(), _ld(a), b.data_ptr(), sb.data_ptr(), _ld(b), M, N, K,
                             out.data_ptr(), _ld(out), _stream(a))
    _check(st, "fp8q_gemm_mx4")
    return out


def _tokens(tokens, device, T=None):
    """tokens checked: int64 [T] on the device; returns T."""
    _vector(tokens, torch.int64, 0, "tokens", device)
    if tokens.dim() != 1 or (T is not None and tokens.numel() != T):
        raise ValueError("tokens must be a vector of one token a row")
    return tokens.numel()


def embedding(weight, tokens, scale=1.0, out=None):
    """Rows of an embedding table, scaled: bf16 out[T, C] = scale weight[tokens], weight
    bf16 or fp32 [V, C], tokens int64 [T].  A token outside the table (padding) gives a row
    of zeros."""
    r = _fast().embedding(weight, tokens, scale, out)
    if r is not None:
        return _done(r, "fp8q_embedding")
    if not isinstance(weight, torch.Tensor) or weight.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("weight must be a 2-D bfloat16 or float32 CUDA tensor")
    _matrix(weight, weight.dtype, "weight")
    T = _tokens(tokens, weight.device)
    V, C = weight.shape
    out = _given(out, torch.bfloat16, "out", (T, C), weight.device)
    st = lib().fp8q_embedding(weight.data_ptr(), 1 if weight.dtype == torch.float32 else 0, V, C, _ld(weight),
                              tokens.data_ptr(), T, float(scale), out.data_ptr(), _ld(out), _stream(weight))
    _check(st, "fp8q_embedding")
    return out


def embedding_backward(dy, tokens, vocab, scale=1.0, dtype=torch.float32, dweight=None, accumulate=False,
                       workspace=None):
    """Gradient of embedding()'s table from that of its output, dy bf16 [T, C]: dweight
    [vocab, C] in `dtype` (float32 or bfloat16), each row the sum of its tokens' rows of dy
    in fp32, times scale, in one order (the same bits on every run); rows of tokens that do
    not occur are zero.  accumulate: dweight (given) is added to, and rows of tokens that do not
    occur stay as they are.  workspace: a uint8 CUDA tensor of
    fp8q_embedding_backward_workspace bytes (a new one when None)."""
    r = _fast().embedding_backward(dy, tokens, vocab, scale, dtype is torch.float32, dweight, accumulate,
                                   workspace) if dtype in (torch.float32, torch.bfloat16) else None
    if r is not None:
        return _done(r, "fp8q_embedding_backward")
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be float32 or bfloat16")
    _matrix(dy, torch.bfloat16, "dy")
    T, C = dy.shape
    _tokens(tokens, dy.device, T)
    if accumulate and dweight is None:
        raise ValueError("accumulate needs the dweight that is added to")
    need = lib().fp8q_embedding_backward_workspace(T, vocab, C)
    if need < 0:
        raise ValueError("invalid number of tokens, vocabulary size or width")
    dweight = _given(dweight, dtype, "dweight", (vocab, C), dy.device)
    workspace = _new_vector(workspace, torch.uint8, need, "workspace", dy.device)
    st = lib().fp8q_embedding_backward(dy.data_ptr(), _ld(dy), tokens.data_ptr(), T, vocab, C, float(scale),
                                       ACCUMULATE if accumulate else 0, dweight.data_ptr(),
                                       1 if dtype is torch.float32 else 0, _ld(dweight), workspace.data_ptr(),
                                       workspace.numel(), _stream(dy))
    _check(st, "fp8q_embedding_backward")
    return dweight


def top_logprobs(logits, tokens, k, temperature=1.0, logp=None, entropy=None, ids=None, top=None, workspace=None):
    """token_logprobs() with each row's k most probable alternatives (k up to MAX_TOP), from one
    read of the logits: returns (logp, entropy, ids, top), ids int64 [T, k] the indices of the
    k largest logits in descending order, equal ones by index, top fp32 [T, k] their
    log-probabilities.  A logit of -inf is no alternative: places left over hold -1 and -inf.  A
    token outside the vocabulary gives 0, 0, ids of -1 and a top of 0.  workspace: a uint8 CUDA
    tensor of fp8q_top_logprobs_workspace bytes (a new one when None and the size needs one)."""
    r = _fast().top_logprobs(logits, tokens, k, temperature, logp, entropy, ids, top, workspace)
    if r is not None:
        return _done(r, "fp8q_top_logprobs")
    if not isinstance(logits, torch.Tensor) or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be a 2-D bfloat16 or float32 CUDA tensor")
    _matrix(logits, logits.dtype, "logits")
    T, V = logits.shape
    dev = logits.device
    _vector(tokens, torch.int64, T, "tokens", dev)
    need = lib().fp8q_top_logprobs_workspace(T, V, k)
    if need < 0:
        raise ValueError("invalid number of tokens, vocabulary size or k")
    logp = _new_vector(logp, torch.float32, T, "logp", dev)
    entropy = _new_vector(entropy, torch.float32, T, "entropy", dev)
    ids = _given(ids, torch.int64, "ids", (T, k), dev)
    top = _given(top, torch.float32, "top", (T, k), dev)
    if not ids.is_contiguous() or not top.is_contiguous():
        raise ValueError("ids and top must be contiguous")
    workspace = _new_vector(workspace, torch.uint8, need, "workspace", dev)
    st = lib().fp8q_top_logprobs(logits.data_ptr(), 1 if logits.dtype == torch.float32 else 0, T, V, _ld(logits),
                                 tokens.data_ptr(), k, float(temperature), logp.data_ptr(), entropy.data_ptr(),
                                 ids.data_ptr(), top.data_ptr(), workspace.data_ptr() if need else None,
                                 workspace.numel(), _stream(logits))
    _check(st, "fp8q_top_logprobs")
    return logp, entropy, ids, top
