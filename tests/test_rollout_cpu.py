"""The 4-bit operators, the embedding and the alternatives without a GPU: their C-ABI's host
code under the sanitizers, their calls through the binding's native code, refusals of the
package's own checks, the rules that choose kernels, the arithmetic that the kernels' indexing rests
on, and that every kernel is launched."""
import ctypes
import os
import random
import re
import subprocess

import pytest
import torch

import paper_2609_22870_amd as fp8q
from paper_2609_22870_amd import _build

import _mx4
import test_binding_cpu as binding
from _ops import F64
from test_binding_cpu import path, stub  # noqa: F401  (fixtures)
from test_sanitizers import CSRC, ROOT, SAN, build_and_run


def test_abi_host_code_under_sanitizers(tmp_path):
    exe = str(tmp_path / "abi_rollout")
    src = os.path.join(ROOT, "paper_2609_22870_amd", "csrc")
    build_and_run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__"] + SAN +
                  ["-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", src,
                   "-x", "c++", os.path.join(src, "abi_rollout.hip"), "-x", "none",
                   os.path.join(CSRC, "abi_rollout_main.cpp"), "-o", exe], exe)


SIZES = binding.SIZES + ("fp8q_embedding_backward_workspace", "fp8q_top_logprobs_workspace")


def bound(path, call):  # noqa: F811
    m = binding.load(path)
    m.bind(tuple(ctypes.cast(getattr(fp8q.lib(), n) if n in SIZES else call, ctypes.c_void_p).value
                 for n in fp8q._NATIVE_API))
    return m


def calls(wrap):
    """(name, arguments, places of given outputs) of ordinary calls, without and with outputs."""
    def new(dtype, *s):
        return wrap(torch.zeros(s, dtype=dtype))

    def u8(*s):
        return new(torch.uint8, *s)

    def f32(*s):
        return new(torch.float32, *s)

    def b16(*s):
        return new(torch.bfloat16, *s)

    def i64(*s):
        return new(torch.int64, *s)

    return [
        ("quantize_mx4", (b16(6, 300), None, None), ()),
        ("quantize_mx4", (b16(6, 300), u8(6, 256), u8(96)), (1, 2)),
        ("dequantize_mx4", (u8(6, 256), u8(96), 300, None), ()),
        ("dequantize_mx4", (u8(6, 256), u8(96), 512, b16(6, 512)), (3,)),
        ("gemm_mx4", (u8(6, 256), u8(96), u8(20, 256), u8(320), None), ()),
        ("gemm_mx4", (u8(6, 256), u8(96), u8(20, 256), u8(320), b16(6, 20)), (4,)),
        ("embedding", (b16(9, 32), i64(5), 1.0, None), ()),
        ("embedding", (f32(9, 32), i64(5), 2.0, b16(5, 32)), (3,)),
        ("embedding_backward", (b16(5, 32), i64(5), 9, 1.0, True, None, False, None), ()),
        ("embedding_backward", (b16(5, 32), i64(5), 9, 1.0, False, b16(9, 32), True, u8(1 << 16)), (5,)),
        ("top_logprobs", (b16(5, 300), i64(5), 4, 1.0, None, None, None, None, None), ()),
        ("top_logprobs", (f32(5, 90000), i64(5), 4, 0.7, f32(5), f32(5), i64(5, 4), f32(5, 4), u8(1 << 21)), (4, 5, 6, 7)),
    ]


def test_ordinary_calls_are_taken(path, stub):  # noqa: F811
    m = bound(path, stub.stub_call)
    count = ctypes.c_int.in_dll(stub, "stub_calls")
    for name, args, given in calls(lambda t: t):
        count.value = 0
        r = getattr(m, name)(*args)
        assert isinstance(r, (tuple, torch.Tensor)) and count.value == 1, name
        outs = [args[i] for i in given]
        assert not outs or all(any(o is g for g in (r if isinstance(r, tuple) else (r,))) for o in outs), name


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
                assert getattr(m, name)(*args[:i], "x", *args[i + 1:]) is None, (name, i)
                if a.dim() == 2:  # one row less
                    assert i == 0 or name == "gemm_mx4" or getattr(m, name)(*args[:i], a[1:], *args[i + 1:]) is None, (name, i)
        assert getattr(m, name)(*args, None) is None, name
    q = dict(a=torch.zeros(6, 256, dtype=torch.uint8), s=torch.zeros(96, dtype=torch.uint8))
    assert m.gemm_mx4(q["a"], q["s"][:95], q["a"], q["s"], None) is None           # scales too short
    assert m.gemm_mx4(q["a"], q["s"], q["a"][:, :128], q["s"], None) is None       # K differs
    assert m.gemm_mx4(q["a"], q["s"], q["a"], q["s"], None) is None                # N = 6: rows with room behind
    assert m.dequantize_mx4(q["a"], q["s"], 513, None) is None
    assert m.dequantize_mx4(q["a"], q["s"], 0, None) is None
    dy, t = torch.zeros(5, 32, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int64)
    assert m.embedding_backward(dy, t, 9, 1.0, True, None, True, None) is None     # nothing to add to
    assert m.embedding_backward(dy, t[:4], 9, 1.0, True, None, False, None) is None
    x = torch.zeros(5, 300)
    assert m.top_logprobs(x, t, 65, 1.0, None, None, None, None, None) is None
    assert m.top_logprobs(x, t, 0, 1.0, None, None, None, None, None) is None
    wide = torch.zeros(5, 8, dtype=torch.int64)
    assert m.top_logprobs(x, t, 4, 1.0, None, None, wide[:, :4], None, None) is None  # rows apart
    assert count.value == 0


def test_the_package_says_what_is_wrong():
    """Calls that the native code leaves end in an error that names the argument (CPU tensors here: the first
    check of each)."""
    b, u, t = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, dtype=torch.int64)
    for call, what in ((lambda: fp8q.quantize_mx4(b), "x must"), (lambda: fp8q.dequantize_mx4(u, u), "codes must"),
                       (lambda: fp8q.gemm_mx4(u, u, u, u), "a must"), (lambda: fp8q.embedding(b, t), "weight must"),
                       (lambda: fp8q.embedding(b.double(), t), "weight must"),
                       (lambda: fp8q.embedding_backward(b, t, 9), "dy must"),
                       (lambda: fp8q.embedding_backward(b, t, 9, dtype=torch.float16), "dtype must"),
                       (lambda: fp8q.top_logprobs(b, t, 2), "logits must"),
                       (lambda: fp8q.top_logprobs(b.half(), t, 2), "logits must")):
        with pytest.raises(ValueError, match=what):
            call()


def test_product_routes():
    """Every size has a kernel that the product launches; one over another at the lines."""
    fn = fp8q.lib().fp8q_gemm_mx4_route
    fn.argtypes, fn.restype = [ctypes.c_int64] * 3, ctypes.c_int
    for M in (1, 16, 33, 64, 128, 200, 500, 1024, 4096, 16384):
        for N in (4, 100, 1000, 4096, 12288, 17408):
            for K in (256, 512, 1024, 4096, 8192, 17408):
                r = fn(M, N, K)
                assert 0 <= r <= 5
                if r == 4:
                    assert K // 256 % 2 == 0
    assert fn(512, 4096, 4096) == 3 and fn(1024, 4096, 4096) == 2      # two 64 x 64 tiles a CU, four
    assert fn(64, 17408, 5120) == 2
    assert fn(4096, 4096, 512) == 0 and fn(4096, 4352, 512) == 1       # whole rounds of large tiles, one more
    assert fn(16384, 12288, 4096) == 0 and fn(8, 12288, 4096) == 5


def test_divisions_by_a_product():
    """embedding.hip's Divisor: n / d for n below 2^36 and d below 2^29, as (n m) >> k."""
    rng = random.Random(4)
    for _ in range(20000):
        d = rng.choice((1, 2, 3, rng.randrange(1, 1 << 29), rng.randrange(1, 5000), 1 << rng.randrange(29)))
        k = 36
        while 1 << (k - 36) < d:
            k += 1
        m = -(-(1 << k) // d)
        assert m < 1 << 64
        q = rng.randrange((1 << 36) // d + 1)
        for n in (q * d, q * d - 1, q * d + d - 1, rng.randrange(1 << 36), (1 << 36) - 1):
            if 0 <= n < 1 << 36:
                assert n * m >> k == n // d and n * m < 1 << 128


def test_sizes_of_workspaces():
    L = fp8q.lib()
    # sorted tokens twice, the bitmap, and two rows of sums a chunk of eight
    assert L.fp8q_embedding_backward_workspace(5003, 32000, 2048) >= 8 * 5003 + 32000 / 8 + 626 * 2 * 2048 * 4
    assert L.fp8q_embedding_backward_workspace(70000, 32000, 64) > 16 * 70000
    assert L.fp8q_top_logprobs_workspace(64, 131072, 20) == 64 * 64 * (16 + 256)
    assert L.fp8q_top_logprobs_workspace(128, 131072, 20) == 0 and L.fp8q_top_logprobs_workspace(1, 1000, 5) == 0


@pytest.mark.parametrize("src", ["mx4.hip", "gemm_mx4.hip", "embedding.hip", "top.hip"])
def test_every_kernel_is_launched(src, tmp_path):
    obj = str(tmp_path / "out.o")
    r = subprocess.run([_build.HIPCC] + _build.FLAGS + _build.EXTRA.get(src, []) +
                       ["-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(_build.CSRC, src), "-o", obj],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = set(re.findall(r"Function Name: (\S+)", r.stderr))
    symbols = {line.split()[-1] for line in
               subprocess.run(["nm", obj], capture_output=True, text=True, check=True).stdout.splitlines()}
    assert kernels and not kernels - symbols, sorted(kernels - symbols)


def test_mxfp4_reference():
    """The 64-bit reference that the GPU tests compare with, on values worked out by hand, and its layout there
    and back."""
    x = torch.zeros(2, 40, dtype=torch.bfloat16)
    # amax 7 (exponent 2, S = 1): ties to even codes, 7 to 6; a unit of zeros; a short last unit
    x[0, :8] = torch.tensor([7.0, 0.25, 0.75, 1.25, 2.5, 3.5, 5.0, -1.75])
    x[0, 32:40] = torch.tensor([-0.0, 2.0 ** -130, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0])
    codes, scales = _mx4.quantize(x)
    assert codes[0, :8].tolist() == [7, 0, 2, 2, 4, 6, 6, 8 + 4] and scales[0, 0] == 127
    assert codes[0, 32] == 8 and scales[0, 1] == 0 and codes[0, 33] == 0  # 2^-130 over 2^-127: 0.125
    assert scales[1].tolist() == [127] * 8 and codes.shape == (2, 256)
    c, s = _mx4.unpacked(*_mx4.packed(codes, scales))
    assert torch.equal(c, codes) and torch.equal(s, scales)
    v = _mx4.values(codes, scales)
    assert v[0, :8].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 4.0, 4.0, -2.0] and v.dtype == F64
