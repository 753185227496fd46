"""MXFP4: quantizer, values and product against 64-bit references.

The quantizer's results are exact: x / S is, so its codes and scale bytes are compared bit for
bit, and so are the values, which bf16 holds.

The product's tolerance.  Products of codes are exact, and so are the sums of those that share
both scales as long as the instruction aligns them in 8 bits or more (36 against 1/4).  An instruction adds the
four 32-deep pieces of 128 (or the eight halves of them) and its accumulator, each sum rounded or
cut to fp32: at most nine times 2^-23 of sum |a b|.  K / 128 instructions in a row, and up to nine sums where
waves share K, give f = (9 K / 128 + 9) 2^-23 of it; then the output's rounding to bf16."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

import _mx4
from _ops import DEV, F64, bf16_half, same, strided, within

pytestmark = pytest.mark.gpu


def check_quantized(x, codes, scales, what):
    want_c, want_s = _mx4.quantize(x.cpu())
    got_c, got_s = _mx4.unpacked(codes, scales)
    bad = got_s != want_s
    assert not bool(bad.any()), (what, "scales", got_s[bad][:5], want_s[bad][:5])
    live = (want_s != 255).repeat_interleave(32, dim=1)
    bad = (got_c != want_c) & live
    assert not bool(bad.any()), (what, "codes", got_c[bad][:5], want_c[bad][:5], int(bad.sum()))


def test_every_value_at_every_scale():
    """Every bf16 magnitude within 2^9 of a unit's largest, of both signs, under every scale byte
    that finite values have; the largest with every mantissa."""
    bits = []
    for field in range(0, 255):  # exponent field of the unit's largest
        lo = max(0, field - 8) << 7
        v = torch.arange(lo, (field + 1) << 7, dtype=torch.int32)
        v = torch.cat((v, v | 0x8000))
        v = torch.nn.functional.pad(v, (0, -len(v) % 31)).view(-1, 31)
        top = (field << 7) + 127 - torch.arange(len(v), dtype=torch.int32) % 128
        v = torch.where((v & 0x7FFF) > top[:, None], top[:, None], v)
        bits.append(torch.cat((v, top[:, None]), dim=1))
    u = torch.cat(bits)
    u = torch.nn.functional.pad(u, (0, 0, 0, -len(u) % 8)).to(torch.int32)
    x = (u - ((u >= 0x8000).int() << 16)).to(torch.int16).view(torch.bfloat16).view(-1, 256)
    codes, scales = fp8q.quantize_mx4(x.to(DEV))
    check_quantized(x, codes, scales, "sweep")
    # and back: exact, and the codes of the values are the codes
    y = fp8q.dequantize_mx4(codes, scales)
    want = _mx4.values(*_mx4.unpacked(codes, scales))
    assert bool((y.cpu().to(F64) == want).all())
    assert bool((torch.signbit(y.cpu()) == (_mx4.unpacked(codes, scales)[0] >= 8)).all())


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 33), (5, 255), (2, 256), (33, 257), (31, 511), (64, 512),
                                       (7, 513), (129, 1000), (40, 4096), (1001, 1037)])
@pytest.mark.parametrize("wide", [False, True])
def test_shapes(rows, cols, wide):
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = (torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g))).bfloat16()
    x[rows // 2, : cols // 2] = 0.0
    x = x.to(DEV)
    given = None
    if wide:
        x = strided(x, 8 - cols % 8 + 8)
        given = torch.full((rows, _mx4.padded(cols) // 2 + 16), 0xAA, dtype=torch.uint8, device=DEV)
    out = None if given is None else given[:, : _mx4.padded(cols) // 2]
    codes, scales = fp8q.quantize_mx4(x, codes=out)
    check_quantized(x, codes, scales, (rows, cols))
    if wide:
        assert bool((given[:, _mx4.padded(cols) // 2:] == 0xAA).all())
    want = _mx4.values(*_mx4.unpacked(codes, scales))
    for n in {1, cols, _mx4.padded(cols)}:
        wide_y = torch.full((rows, n + 3 + 8 * wide), 7.0, dtype=torch.bfloat16, device=DEV)
        y = fp8q.dequantize_mx4(codes, scales, n, out=wide_y[:, :n])
        assert bool((y.cpu().to(F64) == want[:, :n]).all()) and bool((wide_y[:, n:] == 7.0).all())
    assert bool((fp8q.dequantize_mx4(codes, scales).cpu().to(F64) == want).all())


def test_unaligned_rows():
    g = torch.Generator(device=DEV).manual_seed(3)
    flat = torch.randn(40 * 601 + 1, generator=g, device=DEV).bfloat16()
    x = flat[1:].view(40, 601)[:, :600]
    codes, scales = fp8q.quantize_mx4(x)
    check_quantized(x, codes, scales, "unaligned")


def test_not_finite():
    """A NaN or an infinity makes its unit NaN, and the outputs that it enters; the others stay."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(20, 300, generator=g).bfloat16()
    x[3, 40], x[7, 299], x[9, 0] = float("nan"), float("inf"), float("-inf")
    w = torch.randn(48, 300, generator=g).bfloat16()
    codes, scales = fp8q.quantize_mx4(x.to(DEV))
    check_quantized(x, codes, scales, "not finite")
    y = fp8q.dequantize_mx4(codes, scales, 300).cpu()
    nan = torch.zeros(20, 300, dtype=torch.bool)
    nan[3, 32:64] = nan[7, 288:] = nan[9, :32] = True
    assert bool((torch.isnan(y) == nan).all())
    out = fp8q.gemm_mx4(codes, scales, *fp8q.quantize_mx4(w.to(DEV))).cpu()
    rows = torch.isnan(out).all(dim=1)
    assert sorted(torch.nonzero(rows)[:, 0].tolist()) == [3, 7, 9] and bool(torch.isfinite(out[~rows]).all())


def route(M, N, K):
    fn = fp8q.lib().fp8q_gemm_mx4_route
    import ctypes
    fn.argtypes, fn.restype = [ctypes.c_int64] * 3, ctypes.c_int
    return fn(M, N, K)


def operand(rows, K, seed, spread=6):
    codes, scales = _mx4.random_operand(rows, K, seed, spread)
    return (codes, scales) + tuple(t.to(DEV) for t in _mx4.packed(codes, scales))


def check_product(a, b, M, N, K, what, out=None):
    """Against the product in 64 bits (on the GPU: sums of a thousand terms in 53 bits)."""
    c = fp8q.gemm_mx4(a[2], a[3], b[2], b[3], out=out)
    va, vb = _mx4.values(a[0], a[1]).to(DEV), _mx4.values(b[0], b[1]).to(DEV)
    vt = vb.t().contiguous()
    ref, absum = (va @ vt).cpu(), (va.abs() @ vt.abs()).cpu()
    f = (9 * K / 128 + 9) * 2.0 ** -23
    within(c, ref, f * absum + bf16_half(ref.abs() + f * absum), what)
    return c


SIZES = [(1, 4, 256), (1, 16, 512), (7, 36, 256), (16, 16, 2560), (17, 100, 768), (8, 4096, 4096), (33, 1000, 2048),
         (64, 5120, 1280), (100, 132, 5376), (129, 260, 256), (250, 1024, 4352), (256, 4096, 512), (500, 700, 1024),
         (1000, 1028, 768), (1030, 2052, 512), (2050, 2300, 256), (3001, 4100, 1536), (4096, 4096, 512),
         (192, 8192, 256), (1024, 4096, 1024), (5000, 4608, 256)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(M, N, K):
    print("mx4 product", M, N, K, "route", route(M, N, K), flush=True)
    a, b = operand(M, K, 11), operand(N, K, 12)
    c = check_product(a, b, M, N, K, (M, N, K))
    same(c, fp8q.gemm_mx4(a[2], a[3], b[2], b[3]), "two runs")


def test_every_route_is_met():
    assert {route(*s) for s in SIZES} >= {0, 1, 2, 3, 4, 5}, {s: route(*s) for s in SIZES}


@pytest.mark.parametrize("M,N,K", [(20, 256, 256), (256, 512, 256), (300, 20, 768), (768, 768, 768), (2048, 4096, 2048)])
def test_places(M, N, K):
    """Rows of A with one element of a power of two each: C holds the values of B, shifted, exactly, so
    that every code, every scale byte and every place along K shows by itself."""
    codes = torch.zeros(M, K, dtype=torch.uint8)
    g = torch.Generator().manual_seed(5)
    at = torch.randperm(max(M, K), generator=g)[:M] % K
    codes[torch.arange(M), at] = 2  # 1.0
    scales = torch.randint(97, 157, (M, K // 32), generator=g)
    b = operand(N, K, 13, spread=20)
    pa, ps = (t.to(DEV) for t in _mx4.packed(codes, scales))
    c = fp8q.gemm_mx4(pa, ps, b[2], b[3]).cpu().to(F64)
    vb = _mx4.values(b[0], b[1])
    want = vb.t()[at] * torch.exp2(scales[torch.arange(M), at // 32].to(F64) - 127)[:, None]
    assert bool((c == want).all())


def test_strides_and_given_output():
    M, N, K = 200, 520, 1024
    a, b = operand(M, K, 14), operand(N, K, 15)
    want = fp8q.gemm_mx4(a[2], a[3], b[2], b[3])
    sa, sb = strided(a[2], 48), strided(b[2], 16)
    for extra in (4, 8):
        wide = torch.full((M, N + extra), 3.0, dtype=torch.bfloat16, device=DEV)
        got = fp8q.gemm_mx4(sa, a[3], sb, b[3], out=wide[:, :N])
        same(got, want, "strided")
        assert bool((wide[:, N:] == 3.0).all())


def test_layer_of_ragged_width():
    """x of 1000 columns: the zeros that fill its rows up take no part."""
    g = torch.Generator().manual_seed(6)
    x, w = torch.randn(77, 1000, generator=g).bfloat16(), (0.02 * torch.randn(300, 1000, generator=g)).bfloat16()
    qx, qw = fp8q.quantize_mx4(x.to(DEV)), fp8q.quantize_mx4(w.to(DEV))
    c = fp8q.gemm_mx4(*qx, *qw)
    vx, vw = _mx4.values(*_mx4.quantize(x))[:, :1000], _mx4.values(*_mx4.quantize(w))[:, :1000]
    ref, absum = vx @ vw.t(), vx.abs() @ vw.abs().t()
    f = (9 * 8 + 9) * 2.0 ** -23
    within(c, ref, f * absum + bf16_half(ref.abs() + f * absum), "ragged layer")


@pytest.mark.parametrize("M,N,K", [(64, 5120, 2816), (49, 5076, 4352), (100, 5220, 9984), (250, 2300, 13056)])
def test_three_strips(M, N, K):
    """Thin tiles of 48 columns."""
    assert route(M, N, K) == 5
    print("mx4 product", M, N, K, flush=True)
    a, b = operand(M, K, 21), operand(N, K, 22)
    c = check_product(a, b, M, N, K, (M, N, K))
    same(c, fp8q.gemm_mx4(a[2], a[3], b[2], b[3]), "two runs")


@pytest.mark.parametrize("M,N,K", [(5, 3, 256), (1, 1001, 4096), (40, 1, 768), (70, 5075, 2816), (500, 701, 1024), (1030, 2050, 256),
                                   (192, 8189, 256), (2050, 2302, 256), (4090, 4097, 512), (256, 4094, 512), (100, 130, 5376)])
def test_any_number_of_outputs(M, N, K):
    """N that is no multiple of 4: a new output has room behind its rows, and nothing is written there."""
    print("mx4 product", M, N, K, "route", route(M, N, K), flush=True)
    a, b = operand(M, K, 23), operand(N, K, 24)
    c = check_product(a, b, M, N, K, (M, N, K))
    wide = torch.full((M, -(-N // 4) * 4 + 4), 3.0, dtype=torch.bfloat16, device=DEV)
    same(fp8q.gemm_mx4(a[2], a[3], b[2], b[3], out=wide[:, :N]), c, "given")
    assert bool((wide[:, N:] == 3.0).all())
    if N % 4:
        with pytest.raises(fp8q.Fp8qError):
            fp8q.gemm_mx4(a[2], a[3], b[2], b[3], out=torch.empty(M, N, dtype=torch.bfloat16, device=DEV))
