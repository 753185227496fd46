"""The operators around the FP8 layers without a GPU: their C-ABI's host code
under the sanitizers, their calls through the binding's native code, the rules
that choose a gated product's kernel, and the formulas of the gradients that the
GPU tests hold the kernels to, against differences."""
import ctypes
import os

import pytest
import torch

import paper_2609_22870_amd as fp8q

import test_binding_cpu as binding
from _ops import F64, gated_route
from test_binding_cpu import path, stub  # noqa: F401  (fixtures)
from test_sanitizers import CSRC, ROOT, SAN, build_and_run


def test_abi_host_code_under_sanitizers(tmp_path):
    exe = str(tmp_path / "abi_ops")
    src = os.path.join(ROOT, "paper_2609_22870_amd", "csrc")
    build_and_run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__"] + SAN +
                  ["-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", src,
                   "-x", "c++", os.path.join(src, "abi_ops.hip"), "-x", "none",
                   os.path.join(CSRC, "abi_ops_main.cpp"), "-o", exe], exe)


SIZES = binding.SIZES + ("fp8q_rmsnorm_backward_workspace", "fp8q_gemm_gated_workspace", "fp8q_policy_loss_workspace")


def bound(path, call):  # noqa: F811
    m = binding.load(path)
    m.bind(tuple(ctypes.cast(getattr(fp8q.lib(), n) if n in SIZES else call, ctypes.c_void_p).value
                 for n in fp8q._NATIVE_API))
    return m


def calls(wrap):
    """(name, arguments, places of given outputs) of ordinary calls of every
    function, without and with outputs."""
    def new(dtype, *s):
        return wrap(torch.zeros(s, dtype=dtype))

    def u8(*s):
        return new(torch.uint8, *s)

    def f32(*s):
        return new(torch.float32, *s)

    def b16(*s):
        return new(torch.bfloat16, *s)

    x, r, w = b16(6, 256), b16(6, 256), b16(256)
    gated = (u8(40, 256), f32(80), u8(512, 256), f32(8), True)
    logits, tokens, per = b16(5, 300), new(torch.int64, 5), [f32(5) for _ in range(5)]
    loss = (logits, tokens, per[0], per[1], per[2], 0.8, 1.2, 0.1)
    return [
        ("rmsnorm", (x, w, 1e-6, None, None, None, None), ()),
        ("rmsnorm", (x, f32(256), 1e-6, r, b16(6, 256), b16(6, 256), f32(6)), (4, 5, 6)),
        ("rmsnorm_quantize", (x, w, 1e-6, fp8q.BLOCK_1x128, 0, None, None, None, None, None), ()),
        ("rmsnorm_quantize", (x, w, 1e-6, fp8q.ROW, 2, r, u8(6, 256), f32(6), b16(6, 256), f32(6)), (6, 7, 8, 9)),
        ("rmsnorm_backward", (x, r, f32(6), w, None, None, None, None), ()),
        ("rmsnorm_backward", (x, r, f32(6), w, b16(6, 256), b16(6, 256), f32(256), u8(6 * 256 * 4)), (5, 6)),
        ("gemm_gated", gated + (None, None), ()),
        ("gemm_gated", gated + (b16(40, 256), b16(40, 512)), (5, 6)),
        ("gemm_gated_quantized", gated + (None, None, None, None), ()),
        ("gemm_gated_quantized", gated + (u8(40, 256), f32(80), b16(40, 512), u8(40 * 256 * 2)), (5, 6, 7)),
        ("gated_backward", (b16(40, 256), b16(40, 512), 0, None, None, None, None), ()),
        ("gated_backward", (b16(40, 256), b16(40, 512), 4, u8(40, 512), f32(160), u8(512, 128), f32(512)), (3, 4, 5, 6)),
        ("requantize_transposed", (u8(40, 256), f32(80), 0, None, None), ()),
        ("requantize_transposed", (u8(40, 256), f32(80), 2, u8(256, 128), f32(256)), (3, 4)),
        ("token_logprobs", (logits, tokens, 1.0, None, None, None), ()),
        ("token_logprobs", (f32(5, 300), tokens, 0.7, f32(5), f32(5), u8(1 << 16)), (3, 4)),
        ("policy_loss", loss + (None, None, 1.0, None, None, None, None, None, None), ()),
        ("policy_loss", loss + (per[3], per[4], 1.0, u8(80), f32(1), b16(5, 300), f32(5), f32(5), u8(1 << 16)),
         (12, 13, 14, 15)),
    ]


def test_ordinary_calls_are_taken(path, stub):  # noqa: F811
    m = bound(path, stub.stub_call)
    count = ctypes.c_int.in_dll(stub, "stub_calls")
    for name, args, given in calls(lambda t: t):
        count.value = 0
        r = getattr(m, name)(*args)
        assert isinstance(r, tuple) and count.value == 1, name
        outs = [args[i] for i in given]
        assert not outs or all(any(o is g for g in r) for o in outs), name
    # without a residual h is x itself; without `save` there is no pre
    name, args, _ = calls(lambda t: t)[0]
    assert m.rmsnorm(*args)[1] is args[0]
    name, args, _ = calls(lambda t: t)[6]
    assert m.gemm_gated(*args[:4], False, None, None)[1] is None


def test_other_calls_are_left(path, stub):  # noqa: F811
    m = bound(path, stub.stub_call)
    count = ctypes.c_int.in_dll(stub, "stub_calls")
    count.value = 0
    for name, args, _ in calls(lambda t: t.as_subclass(binding.Sub)):
        assert getattr(m, name)(*args) is None, name
    for name, args, _ in calls(lambda t: t):
        for i, a in enumerate(args):
            if isinstance(a, torch.Tensor):
                wrong = a.t() if a.dim() == 2 else a.double() if a.is_floating_point() else a.to(torch.int16)
                assert getattr(m, name)(*args[:i], wrong, *args[i + 1:]) is None, (name, i)
                if name != "policy_loss" or i != 13:
                    assert getattr(m, name)(*args[:i], "x", *args[i + 1:]) is None, (name, i)
        assert getattr(m, name)(*args, None) is None, name
    assert count.value == 0


def test_gated_routes():
    """Every size has a kernel; one over another at the lines; 8-bit output has no
    workspace exactly where one kernel makes it."""
    for M in (1, 16, 17, 32, 33, 64, 65, 128, 129, 500, 4096, 16384):
        for K in (128, 256, 1024, 4096, 8192):
            for F in (128, 640, 4096, 12288, 17408, 25600):
                name, through = gated_route(M, F, K)
                assert name != "split-K"
                assert through == (fp8q.lib().fp8q_gemm_gated_workspace(M, F, K) == 2 * M * F)
                if name in ("large", "half"):
                    assert not through
                if name.startswith("thin") or name in ("two K groups", "small", "eight waves"):
                    assert through
    assert gated_route(8, 12288, 4096)[0].startswith("thin")
    assert gated_route(32, 17408, 5120)[0] == "thin 32 x 32" and gated_route(33, 17408, 5120)[0] == "small"
    assert gated_route(64, 17408, 5120)[0] == "small" and gated_route(65, 17408, 5120)[0] == "half"
    assert gated_route(128, 17408, 512)[0] == "mid"
    assert gated_route(16384, 12288, 4096) == ("large", False)


def test_sizes_of_workspaces():
    L = fp8q.lib()
    assert L.fp8q_rmsnorm_backward_workspace(3, 4096) == 3 * 4096 * 4
    assert L.fp8q_rmsnorm_backward_workspace(16384, 4096) == 512 * 4096 * 4
    assert L.fp8q_rmsnorm_backward_workspace(16384, 1024) == 512 * 1024 * 4
    assert L.fp8q_rmsnorm_backward_workspace(5, 40000) == -1
    assert L.fp8q_policy_loss_workspace(1, 10) >= 16 + 64 * 16
    assert L.fp8q_policy_loss_workspace(0, 10) == -1


@pytest.mark.parametrize("what", ["norm", "gated", "loss"])
def test_gradient_formulas_against_differences(what):
    """The 64-bit formulas that the GPU tests compare with, each along a random
    direction against a central difference."""
    import test_gpu_s_norm as norm
    import test_gpu_t_gated as gated
    import test_gpu_v_loss as loss
    g = torch.Generator().manual_seed(51)
    e = 1e-6
    if what == "norm":
        x, w = torch.randn(3, 64, generator=g, dtype=F64), torch.randn(64, generator=g, dtype=F64)
        dy, u = torch.randn(3, 64, generator=g, dtype=F64), torch.randn(3, 64, generator=g, dtype=F64)

        def f(x):
            return (dy * x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + 1e-6) * w).sum()

        dx = norm.backward_reference(dy, x, 1.0 / torch.sqrt((x * x).mean(dim=1) + 1e-6), w, None)[0]
        assert abs(float((dx * u).sum() - (f(x + e * u) - f(x - e * u)) / (2 * e))) < 1e-7
    elif what == "gated":
        pre, dh = torch.randn(4, 64, generator=g, dtype=F64), torch.randn(4, 32, generator=g, dtype=F64)
        u = torch.randn(4, 64, generator=g, dtype=F64)

        def f(p):
            return (dh * gated.silu(p[:, :32]) * p[:, 32:]).sum()

        assert abs(float((gated.grads(pre, dh) * u).sum() - (f(pre + e * u) - f(pre - e * u)) / (2 * e))) < 1e-7
    else:
        b = loss.batch(9, 40, torch.float32, seed=52)
        u = torch.randn(9, 40, generator=g, dtype=F64)
        d = [float(loss.reference(dict(b, logits=b["logits"].to(F64) + s * u))["loss"]) for s in (e, -e)]
        assert abs(float((loss.reference(b)["dlogits"] * u).sum()) - (d[0] - d[1]) / (2 * e)) < 1e-7
