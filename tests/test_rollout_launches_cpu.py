"""Sizes that the 4-bit operators, the embedding and the alternatives take can be launched: their real host
code, with the HIP runtime's launch calls replaced by a recorder (tests/csrc/launch_recorder.c), at the largest
sizes of the header's rules.  A launch has fewer than 2^32 threads, and at least one workgroup."""
import json
import os
import subprocess
import sys

import pytest

import paper_2609_22870_amd as fp8q

HERE = os.path.dirname(os.path.abspath(__file__))

SCRIPT = """
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
for name, args in json.load(sys.stdin):
    f = getattr(lib, name)
    f.restype = ctypes.c_int
    st = f(*[ctypes.c_double(a) if isinstance(a, float) else ctypes.c_int64(a) for a in args])
    recorder.recorder_print(b"end %d" % st)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """run(calls) -> for each call its status and its launches, (kernel, workgroups, threads)."""
    so = str(tmp_path_factory.mktemp("recorder") / "librecorder.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-fPIC", "-shared", "-o", so, os.path.join(HERE, "csrc", "launch_recorder.c")],
                   check=True)
    fp8q.lib()

    def run(calls):
        r = subprocess.run([sys.executable, "-c", SCRIPT, so, fp8q.LIB_PATH], input=json.dumps(calls), capture_output=True,
                           text=True, timeout=300)
        assert r.returncode == 0, r.stderr
        out, now = [], []
        for line in r.stdout.splitlines():
            word = line.split()
            if word[0] == "launch":
                g, b = [int(w) for w in word[2:5]], [int(w) for w in word[5:8]]
                groups = g[0] * g[1] * g[2]
                now.append((word[1], groups, groups * b[0] * b[1] * b[2]))
            elif word[0] == "end":
                out.append((int(word[1]), now))
                now = []
        assert len(out) == len(calls)
        return out

    return run


AT = 1 << 20  # a pointer that nothing follows
MOST = (1 << 31) - 1


def wide(n):
    """n rounded up to a leading dimension that any type takes."""
    return -(-n // 16) * 16


def backward(T, V, C, f32=1, accumulate=0):
    return ("fp8q_embedding_backward", [AT, C, AT, T, V, C, 1.0, fp8q.ACCUMULATE * accumulate, AT, f32, C, AT, 1 << 50, 0])


def embedding(T, V, C, f32=0):
    return ("fp8q_embedding", [AT, f32, V, C, C, AT, T, 1.0, AT, C, 0])


def top(T, V, k=5, f32=0):
    return ("fp8q_top_logprobs", [AT, f32, T, V, V, AT, k, 1.0, AT, AT, AT, AT, AT, 1 << 50, 0])


def quantize(rows, cols):
    P = -(-cols // 256) * 256
    return ("fp8q_quantize_mx4", [AT, rows, cols, cols, AT, P // 2, AT, 0])


def dequantize(rows, cols):
    P = -(-cols // 256) * 256
    return ("fp8q_dequantize_mx4", [AT, P // 2, AT, rows, cols, AT, cols, 0])


def gemm(M, N, K, lda=None, ldb=None, ldc=None):
    return ("fp8q_gemm_mx4", [AT, AT, lda or K // 2, AT, AT, ldb or K // 2, M, N, K, AT, ldc or wide(N), 0])


def check(calls, results):
    for call, (status, done) in zip(calls, results):
        assert status == 0 and done, (call, status)
        for name, groups, threads in done:
            assert 1 <= groups and threads < 1 << 32, (call, name, groups, threads)


def test_gradient(launches):
    """T ceil(C / 2048) up to 2^25 and V C below 2^33, on both sides of 256 tokens, from few wide rows to many
    narrow ones."""
    calls = [backward(T, V, C, f32, accumulate)
             for T, V, C in ((1, 1, MOST - 15), (3, 1, MOST - 15), (32, 4, 1 << 30), (64, 7, 1 << 30), (64, 15, 1 << 29),
                             (128, 31, 1 << 28), (255, 63, 1 << 27), (256, 1, 1 << 27), (256, 63, 1 << 27), (256, 1, 1 << 28),
                             (256, 127, 1 << 26), (257, 127, 1 << 26), (512, 1, 1 << 27), (16384, 1, 1 << 22),
                             (16385, 1, 1 << 21), (1 << 20, 1, 1 << 16), ((1 << 22) - 1, (1 << 29) - 1, 16),
                             ((1 << 22) - 1, 7, 16384), (1, (1 << 29) - 1, 16), (256, (1 << 29) - 1, 16))
             for f32 in (0, 1) for accumulate in (0, 1)]
    check(calls, launches(calls))


def test_gradient_paths(launches):
    """Up to 256 tokens are compared with each other, more are sorted; few tokens of rows so wide that the former's
    launch, a workgroup a token and 2048 columns, would have 2^32 threads are sorted, too."""
    sizes = [(256, 1000, 4096, True), (257, 1000, 4096, False), (1, 1, MOST - 15, True), (255, 1, 1 << 27, True),
             (256, 1, (1 << 27) - 2048, True), (256, 1, (1 << 27) - 2032, False), (256, 1, 1 << 27, False),
             (64, 1, 1 << 29, False)]
    for (T, V, C, few), (status, done) in zip(sizes, launches([backward(*s[:3]) for s in sizes])):
        names = " ".join(n for n, _, _ in done)
        assert status == 0 and ("embedding_few_kernel" in names) == few and ("sort_" in names) != few, (T, V, C, names)


def test_gradient_workspace():
    """Tokens that are compared need none to speak of; one token more never needs less."""
    need = fp8q.lib().fp8q_embedding_backward_workspace
    for V, C in ((1, 16), (131072, 4096), (1 << 20, 8176), (1, 1 << 27)):
        sizes = [need(T, V, C) for T in (1, 8, 127, 255, 256, 257, 300)]
        assert sizes == sorted(sizes) and sizes[0] == 16 and all(n > 0 for n in sizes)
        assert (sizes[4] == 16) == (C < 1 << 27) and sizes[5] > 257 * 8


def test_rows(launches):
    calls = [embedding(T, V, C, f32) for T, V, C in ((1, 1, MOST - 15), (4, MOST, 16), (32, 9, MOST - 15), ((1 << 22) - 1, 9, 16384),
                                                     (1 << 14, 9, 1 << 22)) for f32 in (0, 1)]
    check(calls, launches(calls))


def test_alternatives(launches):
    calls = [top(T, V, k, f32) for T, V, k in ((1, 1, 1), ((1 << 22) - 1, 64, 64), (1, MOST, 64), (63, MOST, 5),
                                               ((1 << 22) - 1, MOST, 5), ((1 << 22) - 1, 20000, 5)) for f32 in (0, 1)]
    check(calls, launches(calls))


def test_codes(launches):
    calls = [f(*s) for f in (quantize, dequantize) for s in ((1, 1), (1, MOST), (32 << 23, 512), (1 << 14, 1 << 23), (2000, 513))]
    check(calls, launches(calls))


def test_products(launches):
    """Up to 2^22 tiles of 128 x 128, scales of 2^31 bytes a side, and operands that take several launches."""
    calls = [gemm(*s) for s in ((1, 1, 256), (1, 1, 1 << 20), (128, 1 << 21, 256), (1 << 21, 128, 256), (1 << 18, 1 << 18, 256),
                                (1 << 15, 1 << 15, 1 << 20), (65536, 4, (1 << 20) - 256), ((1 << 28) - 128, 128, 256),
                                (4, 65535, (1 << 20) - 256), (3001, 17408, 5120))]
    check(calls, launches(calls))


UNSUPPORTED = -2
HEADER = os.path.join(os.path.dirname(HERE), "include", "fp8q.h")


def rules(name):
    """What the header says before the declaration of `name`, in one line."""
    text = open(HEADER).read()
    at = text.index("fp8q_status %s(" % name)
    return " ".join(text[text.rindex("/*", 0, at):at].replace("\n *", " ").split())


# (taken, refused, the rule as the header states it)
LIMITS = [
    (gemm(128, 128, 1 << 20, lda=(1 << 23) - 16), gemm(128, 128, 1 << 20, lda=1 << 23), "lda below 2^23"),
    (gemm(128, 128, (1 << 21) - 256, ldb=(1 << 20) - 16), gemm(128, 128, 512, ldb=1 << 20), "ldb below 2^20 (so K below 2^21)"),
    (gemm(128, 128, (1 << 21) - 256), gemm(128, 128, 1 << 21), "ldb below 2^20 (so K below 2^21)"),
    (gemm(128, 128, 512, ldc=(1 << 22) - 4), gemm(128, 128, 512, ldc=1 << 22), "ldc below 2^22"),
    (gemm(1 << 18, 1 << 18, 256), gemm(1 << 18, (1 << 18) + 1, 256), "up to 2^22 tiles of 128 x 128"),
    (gemm((1 << 28) - 1, 1, 256), gemm(1 << 28, 1, 256), "M K / 32 and N K / 32 below 2^31"),
    (embedding(1 << 14, 9, 1 << 22), embedding((1 << 14) + 1, 9, 1 << 22), "ceil(T / 4) ceil(C / 2048) up to 2^23"),
    (embedding((1 << 22) - 1, 9, 16), embedding(1 << 22, 9, 16), "T below 2^22"),
    (backward(1 << 20, 1, 1 << 16), backward(1 << 20, 1, (1 << 16) + 16), "T ceil(C / 2048) up to 2^25"),
    (backward(5, (1 << 29) - 1, 16), backward(5, 1 << 29, 16), "V C below 2^33"),
    (quantize(32 << 23, 512), quantize((32 << 23) + 1, 512), "Up to 2^23 tiles of 32 x 512"),
]


def test_limits(launches):
    """The header's limits are the code's, on both sides, and a refused call launches nothing."""
    results = launches([c for taken, refused, _ in LIMITS for c in (taken, refused)])
    for i, (taken, refused, rule) in enumerate(LIMITS):
        check([taken], results[2 * i:2 * i + 1])
        assert results[2 * i + 1] == (UNSUPPORTED, []), (refused, results[2 * i + 1])
        assert rule in rules(taken[0]), (taken[0], rule)
