"""The MXFP4 product over all scales of E8M0, the bytes 0 and 254 among them.

What a pair of scales comes to is 2^(byte + byte - 254).  Where it is far from what fp32 holds on one side
only (2^-127 times 2^127, say) the product is an ordinary number, and the tolerance that of ordinary products
(test_gpu_za_mx4.py).  Results past bf16's range are infinite; partial sums below 2^-126 are subnormal in fp32,
and a matrix instruction may take them as zeros: 2^-126 for each of the instructions in a row, no more."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

import _mx4
from _ops import DEV, F64, bf16_half, same, within
from test_gpu_za_mx4 import check_product, route

pytestmark = pytest.mark.gpu

# every route, and each of the thin tiles
SIZES = [(1, 4, 256), (8, 4096, 512), (33, 1000, 2048), (64, 5120, 2816), (128, 700, 5376), (192, 1024, 1024), (250, 2300, 13056),
         (500, 700, 1024), (256, 4096, 512), (1030, 2052, 512), (1000, 1028, 1024), (2050, 2300, 512), (3001, 4100, 768), (4096, 4096, 512)]


def operand(rows, K, exponents, seed, codes=None):
    """Codes at random, the scale byte of unit u exponents[:, u]."""
    g = torch.Generator().manual_seed(seed)
    if codes is None:
        codes = torch.randint(0, 16, (rows, K), generator=g).to(torch.uint8)
    scales = exponents.expand(rows, K // 32).contiguous()
    return (codes, scales) + tuple(t.to(DEV) for t in _mx4.packed(codes, scales))


def test_every_route_is_met():
    assert {route(*s) for s in SIZES} >= {0, 1, 2, 3, 4, 5}, {s: route(*s) for s in SIZES}


@pytest.mark.parametrize("M,N,K", SIZES)
def test_far_scales_that_cancel(M, N, K):
    """Unit u of A has the byte p_u and a few more or less, that of B 254 - p_u: every byte is met where K is long
    enough, 0 and 254 in all sizes but the smallest."""
    print("mx4 scales", M, N, K, "route", route(M, N, K), flush=True)
    g = torch.Generator().manual_seed(M + N + K)
    U = K // 32
    p = torch.randint(0, 255, (U,), generator=g)
    p[:4] = torch.tensor([0, 254, 127, 1])
    p[-3:] = torch.tensor([254, 3, 0])
    a = operand(M, K, (p + torch.randint(-3, 4, (M, U), generator=g)).clamp(0, 254), 51)
    b = operand(N, K, (254 - p + torch.randint(-3, 4, (N, U), generator=g)).clamp(0, 254), 52)
    for _, scales, _, _ in (a, b):
        assert M == 1 or (int(scales.min()) == 0 and int(scales.max()) == 254)
    c = check_product(a, b, M, N, K, (M, N, K))
    assert bool(torch.isfinite(c).all())
    same(c, fp8q.gemm_mx4(a[2], a[3], b[2], b[3]), "two runs")


@pytest.mark.parametrize("M,N,K", SIZES)
def test_every_pair_of_scales(M, N, K):
    """One element of 1 in each row of A, of any scale; B of any scale, so that every sum has one term and zeros:
    the value itself where bf16 holds it, infinite past it, and zero or the value below fp32's smallest normal.  The
    zeros' scales are as far, and leave nothing."""
    print("mx4 places", M, N, K, "route", route(M, N, K), flush=True)
    g = torch.Generator().manual_seed(M * N + K)
    U = K // 32
    at = torch.randint(0, K, (M,), generator=g)
    codes = torch.zeros(M, K, dtype=torch.uint8)
    codes[torch.arange(M), at] = 2  # 1.0
    def bytes_of(rows):
        s = torch.randint(0, 255, (rows, U), generator=g)
        ends = torch.randint(0, 6, (rows, U), generator=g)
        return torch.where(ends == 0, torch.zeros_like(s), torch.where(ends == 1, torch.full_like(s, 254), s))
    a = operand(M, K, bytes_of(M), 53, codes)
    b = operand(N, K, bytes_of(N), 54)
    c = fp8q.gemm_mx4(a[2], a[3], b[2], b[3]).cpu().to(F64)
    exact = _mx4.values(b[0], b[1]).t()[at] * torch.exp2(a[1][torch.arange(M), at // 32].to(F64) - 127)[:, None]
    # (E2M1's mantissas fit bf16's: nothing above 2^-126 is rounded)
    over, small = exact.abs() >= 2.0 ** 128, exact.abs() < 2.0 ** -126
    want = torch.where(over, torch.sign(exact) * float("inf"), exact)
    bad = ~small & (c != want)
    assert not bool(bad.any()), (c[bad][:5], want[bad][:5], int(bad.sum()))
    # each of the K / 128 instructions in a row and of the nine sums at the end may cut 2^-126; bf16's own step is less
    assert bool(((c - exact).abs()[small] <= 2.0 ** -126).all())


@pytest.mark.parametrize("M,N,K", [(20, 256, 512), (500, 700, 1024), (4096, 4096, 512)])
def test_layer_of_tiny_and_huge_values(M, N, K):
    """A layer whose activations are near bf16's smallest normals and weights near its largest, through the
    quantizer: the product of what the codes stand for."""
    print("mx4 layer", M, N, K, flush=True)
    g = torch.Generator().manual_seed(M + 7)
    x = (torch.randn(M, K, generator=g) * 2.0 ** -122).bfloat16()
    w = (torch.randn(N, K, generator=g) * 2.0 ** 122).bfloat16()
    qx, qw = fp8q.quantize_mx4(x.to(DEV)), fp8q.quantize_mx4(w.to(DEV))
    vx, vw = _mx4.values(*_mx4.quantize(x)).to(DEV), _mx4.values(*_mx4.quantize(w)).to(DEV)
    vt = vw.t().contiguous()
    ref, absum = (vx @ vt).cpu(), (vx.abs() @ vt.abs()).cpu()
    f = (9 * K / 128 + 9) * 2.0 ** -23
    within(fp8q.gemm_mx4(*qx, *qw), ref, f * absum + bf16_half(ref.abs() + f * absum), "far layer")
