"""Rows so far apart that their offsets pass 32 bits, in elements and in bytes, for each
operand of the 4-bit operators, the embedding and the alternatives: the results of rows that lie
close together."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

import _mx4
from _ops import DEV, same

pytestmark = pytest.mark.gpu

FAR = (1 << 31) - 16  # elements from a row to the next: three rows pass 2^32


def far(x, ld=FAR):
    """x with rows ld elements apart, in memory that holds nothing else (about 2 ld elements a row
    pair are only reserved)."""
    rows, cols = x.shape
    y = torch.empty((rows - 1) * ld + cols, dtype=x.dtype, device=DEV).as_strided((rows, cols), (ld, 1))
    y.copy_(x)
    return y


def rand(rows, cols, dtype=torch.bfloat16, seed=91):
    return torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def test_quantized_and_values():
    x = rand(3, 700)
    codes, scales = fp8q.quantize_mx4(x)
    c, s = fp8q.quantize_mx4(far(x))
    same(c, codes, "codes")
    same(s, scales, "scales")
    c, s = fp8q.quantize_mx4(x, codes=far(torch.zeros_like(codes)))
    same(c.contiguous(), codes, "codes far apart")
    same(s, scales, "scales")
    values = fp8q.dequantize_mx4(codes, scales, 700)
    same(fp8q.dequantize_mx4(c, s, 700), values, "values of codes far apart")
    del c
    same(fp8q.dequantize_mx4(codes, scales, 700, out=far(torch.zeros_like(values))).contiguous(), values, "values")


# (rows that are cut into several launches, each within the kernels' 32-bit offsets; odd row counts there)
@pytest.mark.parametrize("M,N,lda,ldb,ldc", [(1025, 132, (1 << 22) + 16, 256, 132), (40, 4100, 256, (1 << 20) - 16, 4100),
                                             (1300, 260, 256, 256, (1 << 21) + 8), (600, 4100, 1 << 22, 1 << 19, 1 << 21)])
def test_product(M, N, lda, ldb, ldc):
    K = 512
    print("far product", M, N, lda, ldb, ldc, flush=True)
    a, b = (_mx4.random_operand(n, K, seed) for n, seed in ((M, 92), (N, 93)))
    (ca, sa), (cb, sb) = ((t.to(DEV) for t in _mx4.packed(*o)) for o in (a, b))
    out = far(torch.zeros(M, N, dtype=torch.bfloat16, device=DEV), ldc)
    fp8q.gemm_mx4(far(ca, lda), sa, far(cb, ldb), sb, out=out)
    y = out.contiguous().cpu().double()
    va, vb = _mx4.values(*a), _mx4.values(*b)
    # one rounding to bf16, and the additions of 512 products in fp32
    exact = va @ vb.t()
    bound = 2.0 ** -8 * exact.abs() + K * 2.0 ** -23 * (va.abs() @ vb.abs().t())
    assert bool(((y - exact).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_embedding(dtype):
    w, dy = rand(3, 96, dtype), rand(4, 96)
    tokens = torch.tensor([2, 0, 2, 1], device=DEV)
    y = fp8q.embedding(w, tokens, 1.5)
    same(fp8q.embedding(far(w), tokens, 1.5), y, "rows of a far table")
    same(fp8q.embedding(w, tokens, 1.5, out=far(torch.zeros_like(y))).contiguous(), y, "rows far apart")
    tokens[1] = 2  # (row 0 gets zeros)
    dw = fp8q.embedding_backward(dy, tokens, 3, 1.5, dtype=dtype)
    same(fp8q.embedding_backward(far(dy), tokens, 3, 1.5, dtype=dtype), dw, "dy far apart")
    there = far(torch.ones_like(dw))
    fp8q.embedding_backward(dy, tokens, 3, 1.5, dtype=dtype, dweight=there)
    same(there.contiguous(), dw, "a far table's gradient")
    twice = dw.clone()
    for t in (twice, there):
        fp8q.embedding_backward(dy, tokens, 3, 1.5, dtype=dtype, dweight=t, accumulate=True)
    same(there.contiguous(), twice, "added to")


@pytest.mark.parametrize("V", [5000, 100000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_alternatives(V, dtype):
    x = rand(3, V, dtype)
    tokens = torch.tensor([5, V - 1, 0], device=DEV)
    for a, b in zip(fp8q.top_logprobs(far(x), tokens, 9), fp8q.top_logprobs(x, tokens, 9)):
        same(a, b, "alternatives")


def test_large_gradient():
    """A table of just under 2^33 elements, in bf16: rows at its end are summed, filled and left."""
    V, C = (1 << 22) - 1, 2048
    dy, tokens = rand(70, C), torch.tensor([V - 1, V - 2, 7, V - 1, V] * 14, device=DEV)
    dw = torch.ones((V, C), dtype=torch.bfloat16, device=DEV)
    fp8q.embedding_backward(dy, tokens, V, dtype=torch.bfloat16, dweight=dw)
    d = dy.double().view(14, 5, C)
    for row, want in ((V - 1, (d[:, 0] + d[:, 3])), (V - 2, d[:, 1]), (7, d[:, 2])):
        # fp32 sums of up to 28 rows, one rounding to bf16
        exact, most = want.sum(0), want.abs().sum(0)
        assert bool(((dw[row].double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 28 * 2.0 ** -23 * most).all()), row
    for rows in (slice(0, 7), slice(8, 1 << 21), slice(1 << 21, V - 2)):
        assert not bool(dw[rows].any())
