"""RMS norm with the residual's addition, bf16 and FP8 output, and its
gradients, against 64-bit references.

Tolerances.  The row's sum of squares is added from positive terms in fp32, at
most 64 roundings deep (up to 32 in a thread, 10 across it), each 2^-24 of the
whole: rstd, half of it and a few roundings more, is within 40 x 2^-24.  y has
two products more, and a bf16 rounding.  In the backward pass the same
depth bounds the dot product by 64 x 2^-24 of the sum of its terms' magnitudes."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, bf16_half, block_scales, check_units, same, strided, within

pytestmark = pytest.mark.gpu

EPS = 1e-6
U = 2.0 ** -24
REL_RSTD, REL_Y = 40 * U, 44 * U
# one row and a few, every shape of threads and pieces a row takes, its edges
SHAPES = [(1, 16), (3, 128), (5, 512), (2, 528), (9, 1024), (4, 1040), (3, 2048), (300, 4096), (5, 5120), (3, 6144),
          (2, 6160), (2, 8192), (2, 8208), (3, 16384), (2, 32768)]


def inputs(rows, cols, seed, residual=True, f32=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    x[:, ::37] *= 50.0
    w = 1.0 + 0.1 * torch.randn(cols, generator=g)
    r = torch.randn(rows, cols, generator=g).bfloat16() if residual else None
    return x.bfloat16(), w if f32 else w.bfloat16(), r


def reference(x, w, r, eps=EPS):
    """(h in bf16, rstd, y) in 64 bits from the rounded h."""
    h = x if r is None else (x.float() + r.float()).bfloat16()
    v = h.to(F64)
    rstd = 1.0 / torch.sqrt((v * v).mean(dim=1) + eps)
    return h, rstd, v * rstd[:, None] * w.to(F64)


def on(t):
    return None if t is None else t.to(DEV)


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_bf16_output(shape, residual):
    x, w, r = inputs(*shape, seed=1, residual=residual, f32=residual)
    print("norm bf16", shape, residual, flush=True)
    y, h, rstd = fp8q.rmsnorm(on(x), on(w), EPS, residual=on(r))
    hr, rr, yr = reference(x, w, r)
    same(h, hr, "h")
    within(rstd, rr, REL_RSTD * rr, "rstd")
    within(y, yr, bf16_half(yr * (1 + REL_Y)) + REL_Y * yr.abs(), "y")


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] % 128 == 0])
def test_block_output(shape, residual, pow2):
    x, w, r = inputs(*shape, seed=2, residual=residual)
    print("norm 1x128", shape, residual, pow2, flush=True)
    codes, scales, h, rstd = fp8q.rmsnorm_quantize(on(x), on(w), EPS, residual=on(r), pow2=pow2)
    hr, rr, yr = reference(x, w, r)
    same(h, hr, "h")
    within(rstd, rr, REL_RSTD * rr, "rstd")
    check_units(codes, block_scales(scales, *shape), yr, REL_Y, pow2=pow2)


@pytest.mark.parametrize("shape", SHAPES)
def test_row_output(shape):
    x, w, r = inputs(*shape, seed=3)
    print("norm row", shape, flush=True)
    codes, scales, h, _ = fp8q.rmsnorm_quantize(on(x), on(w), EPS, fp8q.ROW, residual=on(r))
    hr, _, yr = reference(x, w, r)
    same(h, hr, "h")
    # one unit a row: pad it to whole runs of 128 for the check, and give every run the row's amax
    pad = -shape[1] % 128
    amax = yr.abs().amax(dim=1, keepdim=True)
    v = torch.cat((yr, torch.zeros(shape[0], pad, dtype=F64)), dim=1).view(shape[0], -1, 128)
    v = torch.cat((amax[:, :, None].expand(-1, v.shape[1], 1), v), dim=2)
    got = torch.cat((codes.cpu(), torch.zeros(shape[0], pad, dtype=torch.uint8)), dim=1).view(shape[0], -1, 128)
    top = torch.full((shape[0], got.shape[1], 1), 0x7e, dtype=torch.uint8)  # 448
    got, n = torch.cat((top, got), dim=2), v.shape[1]
    s = scales.cpu().to(F64)[:, None]
    ok = (s - amax / 448.0).abs() <= (REL_Y + 2 * U) * amax / 448.0
    assert bool(ok.all())
    q, d = v / s[:, :, None], REL_Y + 2.0 ** -22
    val = got.view(torch.float8_e4m3fn).float().to(F64)
    cast = lambda t: t.clamp(-448, 448).float().to(torch.float8_e4m3fn).float().to(F64)  # noqa: E731
    lo, hi = torch.minimum(cast(q * (1 - d)), cast(q * (1 + d))), torch.maximum(cast(q * (1 - d)), cast(q * (1 + d)))
    assert n and bool(((val >= lo) & (val <= hi)).all())


def test_special_rows():
    """A row of zeros (S = 1), one whose squares are below eps, weights so small
    that a unit's scale is below 2^-90, and subnormal: every path of the cast."""
    x, w, _ = inputs(6, 512, seed=4, residual=False, f32=True)
    x[1] = 0
    x[2] = (x[2].float() * 1e-12).bfloat16()
    w[128:256] *= 2.0 ** -100
    w[256:384] *= 2.0 ** -138
    w[384:] = 0.0
    codes, scales, h, rstd = fp8q.rmsnorm_quantize(on(x), on(w), EPS)
    _, rr, yr = reference(x, w, None)
    within(rstd, rr, REL_RSTD * rr, "rstd")
    s = block_scales(scales, 6, 512)
    yf = yr.float().to(F64)  # (subnormal values are what fp32 holds)
    check_units(codes[:, :256], s[:, :256], yr[:, :256], REL_Y)
    # units near 2^-138: fp32 holds them to 2^-149 absolutely, so the bounds are on that
    sub = s[:, 256:384:128]
    amax = yf[:, 256:384].abs().amax(dim=1, keepdim=True)
    assert bool(((sub - amax / 448).abs() <= 2.0 ** -149 + 1e-5 * amax / 448).logical_or((sub == 1)).all())
    assert bool((s[:, 384:] == 1).all()) and not (codes[:, 384:] & 0x7f).any()
    assert bool((s[1] == 1).all()) and not (codes[1] & 0x7f).any()


@pytest.mark.parametrize("into", ["x", "residual"])
def test_h_in_place_strides_and_stream(into):
    """h over x or over the residual, rows further apart than they are long,
    outputs given, on a stream of its own."""
    x, w, r = inputs(67, 5120, seed=5)
    want = fp8q.rmsnorm_quantize(on(x), on(w), EPS, residual=on(r))
    gx, gr = strided(on(x), 24), strided(on(r), 8)
    codes = torch.zeros(67, 5136, dtype=torch.uint8, device=DEV)[:, :5120]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = fp8q.rmsnorm_quantize(gx, on(w), EPS, residual=gr, codes=codes, h=gx if into == "x" else gr)
    torch.cuda.synchronize()
    assert got[0] is codes and got[2] is (gx if into == "x" else gr)
    for a, b, n in zip(got, want, ("codes", "scales", "h", "rstd")):
        same(a, b, n)


def backward_reference(dy, h, rstd, w, dres):
    dy, h, rstd, w = dy.to(F64), h.to(F64), rstd.to(F64)[:, None], w.to(F64)
    xhat, g = h * rstd, dy * w
    n = h.shape[1]
    dx = rstd * (g - xhat * (g * xhat).mean(dim=1, keepdim=True))
    # what fp32 may lose before the last rounding
    lost = rstd * (4 * U * g.abs() + xhat.abs() * (64 * U * (g * xhat).abs().sum(dim=1, keepdim=True) / n
                                                   + 6 * U * (g * xhat).mean(dim=1, keepdim=True).abs()))
    if dres is not None:
        dx = dx + dres.to(F64)
        lost = lost + 2 * U * dx.abs()
    return dx, lost, (dy * xhat).sum(dim=0), (dy * xhat).abs().sum(dim=0)


@pytest.mark.parametrize("rows", [1, 5, 1500])
@pytest.mark.parametrize("cols,dres,f32", [(16, True, False), (512, True, True), (1024, False, False), (2048, True, True),
                                           (4096, True, False), (5120, False, True), (8192, True, False),
                                           (16384, True, False), (32768, False, True)])
def test_backward(rows, cols, dres, f32):
    if rows * cols > 2 ** 23:
        rows = 300
    print("norm backward", rows, cols, flush=True)
    x, w, _ = inputs(rows, cols, seed=6, residual=False, f32=f32)
    g = torch.Generator().manual_seed(7)
    dy = (1e-3 * torch.randn(rows, cols, generator=g)).bfloat16()
    dr = (1e-3 * torch.randn(rows, cols, generator=g)).bfloat16() if dres else None
    rstd = (1.0 / torch.sqrt((x.to(F64) ** 2).mean(dim=1) + EPS)).float()
    dx, dw = fp8q.rmsnorm_backward(on(dy), on(x), on(rstd), on(w), dres=on(dr))
    ref, lost, wr, wabs = backward_reference(dy, x, rstd, w, dr)
    within(dx, ref, bf16_half(ref.abs() + lost) + lost + 1e-40, "dx")
    # a column's terms: at most rows / 256 in a thread, 512 parts in 32 runs of 16 and those: below 64 roundings
    # deep, but rows / walkers for many rows
    within(dw, wr, (64 + rows / 256) * U * wabs + 1e-40, "dweight")
    again = fp8q.rmsnorm_backward(on(dy), on(x), on(rstd), on(w), dres=on(dr))
    same(dx, again[0], "dx of two runs")
    same(dw, again[1], "dweight of two runs")


def test_backward_against_differences():
    """sum(dx u) and sum(dw v) against central differences of L = sum(dy y(x, w))
    in 64 bits along u and v.  The difference's own error is of third order in its
    step (1e-4); dx is rounded to bf16, at most 2^-8 of every term, and
    4480 independent roundings add up as the root of their squares (4 times it)."""
    x, w, _ = inputs(7, 640, seed=8, residual=False, f32=True)
    g = torch.Generator().manual_seed(9)
    dy = torch.randn(7, 640, generator=g).bfloat16()
    u, v = torch.randn(7, 640, generator=g, dtype=F64), torch.randn(640, generator=g, dtype=F64)
    rstd = (1.0 / torch.sqrt((x.to(F64) ** 2).mean(dim=1) + EPS)).float()
    dx, dw = fp8q.rmsnorm_backward(on(dy), on(x), on(rstd), on(w))

    def loss(xx, ww):
        return (dy.to(F64) * (xx / torch.sqrt((xx * xx).mean(dim=1, keepdim=True) + EPS) * ww)).sum()

    e = 1e-4
    along_u = (loss(x.to(F64) + e * u, w.to(F64)) - loss(x.to(F64) - e * u, w.to(F64))) / (2 * e)
    along_v = (loss(x.to(F64), w.to(F64) + e * v) - loss(x.to(F64), w.to(F64) - e * v)) / (2 * e)
    dx, dw = dx.cpu().to(F64), dw.cpu().to(F64)
    assert abs(float((dx * u).sum() - along_u)) <= 4 * 2.0 ** -8 * float((dx * u).pow(2).sum().sqrt()) + 1e-5
    assert abs(float((dw * v).sum() - along_v)) <= 1e-5 * float((dw * v).abs().sum()) + 1e-7


def test_backward_in_place_and_workspace():
    x, w, _ = inputs(130, 4096, seed=10, residual=False)
    dy, dr = (torch.randn(130, 4096) * 1e-3).bfloat16(), (torch.randn(130, 4096) * 1e-3).bfloat16()
    rstd = (1.0 / torch.sqrt((x.to(F64) ** 2).mean(dim=1) + EPS)).float()
    want = fp8q.rmsnorm_backward(on(dy), on(x), on(rstd), on(w), dres=on(dr))
    ws = torch.full((fp8q.lib().fp8q_rmsnorm_backward_workspace(130, 4096),), 0xff, dtype=torch.uint8, device=DEV)
    for over in ("dy", "dres"):
        t = {"dy": strided(on(dy), 8), "dres": strided(on(dr), 16)}
        got = fp8q.rmsnorm_backward(t["dy"], on(x), on(rstd), on(w), dres=t["dres"], dx=t[over], workspace=ws)
        assert got[0] is t[over]
        same(got[0], want[0], over)
        same(got[1], want[1], "dweight")


def test_rows_past_32_bits():
    """Rows that start past 2^31 elements of a buffer."""
    cols, rows, ld = 4096, 700, 1 << 22
    x, w, _ = inputs(rows, cols, seed=11, residual=False)
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device=DEV).view(rows, ld)
    far = buf[:, :cols]
    far.copy_(x)
    a, b = fp8q.rmsnorm_quantize(far, on(w), EPS), fp8q.rmsnorm_quantize(on(x), on(w), EPS)
    for s, t in zip((a[0], a[1], a[3]), (b[0], b[1], b[3])):
        same(s, t, "rows far apart")


@pytest.mark.parametrize("f", ["rmsnorm", "rmsnorm_quantize"])
def test_refusals(f):
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(256, dtype=torch.bfloat16, device=DEV)
    call = getattr(fp8q, f)
    for bad in (lambda: call(x.float(), w, EPS), lambda: call(x[0], w, EPS), lambda: call(x, w[:128], EPS),
                lambda: call(x, w.double(), EPS), lambda: call(x, w, EPS, residual=x[:2]),
                lambda: call(x, w, EPS, h=x), lambda: call(x.cpu(), w, EPS), lambda: call(x.t(), w, EPS)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: call(x, w, -1.0), -1), (lambda: call(x, w, float("nan")), -1),
                        (lambda: call(x[:, :136], w[:136].clone(), EPS), -2),
                        (lambda: call(x[:, 1:129], w[:128], EPS), -3)):
        with pytest.raises(fp8q.Fp8qError) as e:
            bad()
        assert e.value.status == status
    if f == "rmsnorm_quantize":
        for g, status in ((fp8q.BLOCK_128x128, -2), (fp8q.COL, -2)):
            with pytest.raises((fp8q.Fp8qError, ValueError)):
                call(x, w, EPS, g)
        with pytest.raises(fp8q.Fp8qError):
            call(x[:, :144], w[:144].clone(), EPS)  # no whole 1x128 units
