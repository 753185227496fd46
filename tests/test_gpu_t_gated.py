"""The gated feed-forward block: silu(X Wg^T) * (X Wu^T) from FP8 operands on
every kernel it can take, with and without kept pre-activations, in bf16 and in
8 bits; and the gradients of its pre-activations in both FP8 layouts.

Tolerances.  The kept pre-activations are a GEMM's output and are held to the
model of the matrix instruction (tests/csrc/mfma_model.c) as fp8q_gemm's are.  H
is held to the 64-bit silu(g) u over the interval that the model leaves for g and
u, with 2^-18 more of its value for exp and the reciprocal (|g| 2^-24 and a few
units; |g| is below 40 here), then half a bf16 unit."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_22870_amd as fp8q
from paper_2609_22870_amd import synth

import _par
from _ops import DEV, F64, bf16_half, block_scales, check_units, gated_route, same, strided, values, within

pytestmark = pytest.mark.gpu

B1, B128 = fp8q.BLOCK_1x128, fp8q.BLOCK_128x128

# (M, K, F): (kernel, whether 8-bit output goes through bf16): one row, ragged rows, odd numbers of K blocks; large
# tiles with a last round whole, in halves and in quarters
ROUTES = {
    (1, 128, 128): ("thin 16 x 32", True),
    (8, 1152, 1024): ("thin 16 x 32", True),
    (13, 640, 17408): ("thin 16 x 32", True),
    (30, 640, 16512): ("thin 32 x 32", True),
    (61, 1152, 1152): ("thin 32 x 32", True),
    (30, 1280, 8064): ("thin 32 x 64", True),
    (121, 1920, 2048): ("thin 32 x 64", True),
    (50, 1152, 8192): ("thin 64 x 64", True),
    (61, 256, 8192): ("two K groups", True),
    (250, 256, 1152): ("two K groups", True),
    (50, 640, 17408): ("small", True),
    (300, 128, 1152): ("small", True),
    (200, 1280, 4096): ("eight waves", True),
    (250, 384, 6528): ("eight waves", True),
    (700, 640, 8064): ("mid", True),
    (300, 640, 6528): ("mid", False),
    (200, 1280, 8320): ("half", False),
    (200, 640, 16512): ("large", False),
    (2500, 1152, 8192): ("large", False),
    (2500, 2048, 2048): ("large", False),
    (4096, 1152, 2176): ("large", False),
    (4353, 1152, 2304): ("mid", True),
}


def operands(M, K, F, seed, sigma=None):
    x = synth.activations(M, K, seed=seed, outlier_seed=seed + 1, device=DEV)
    w = synth.weights(2 * F, K, seed=seed + 2, device=DEV)
    if sigma is not None:
        w = (w.float() * (sigma / synth.SIGMA_W)).bfloat16()
    return fp8q.quantize(x, B1) + fp8q.quantize(w, B128)


def silu(g):
    return g / (1.0 + torch.exp(-g))


@pytest.mark.parametrize("shape", list(ROUTES))
def test_every_kernel_against_the_model(shape):
    M, K, F = shape
    assert gated_route(M, F, K) == ROUTES[shape]
    print("gated", shape, ROUTES[shape], flush=True)
    A, sA, B, sB = operands(M, K, F, seed=901)
    h, pre = fp8q.gemm_gated(A, sA, B, sB, save=True)
    # a sample of rows (edges of tiles) and of columns of both weights
    rows = np.unique(np.r_[0, M - 1, np.arange(0, M, 1 + M // 24)])
    cols = np.unique(np.r_[0, F - 1, np.arange(0, F, 1 + F // 60), np.arange(min(F, 130) - 4, min(F, 130))])
    n = np.r_[cols, cols + F]
    a, b = A.cpu().numpy()[rows], B.cpu().numpy()[n]
    sa = sA.cpu().numpy().reshape(K // 128, M)[:, rows].reshape(-1)
    # 128 x 128 scales per row of the sample, as 1x128 ones
    sb = sB.cpu().numpy().reshape(2 * F // 128, K // 128)[n // 128].T.reshape(-1)
    model, absum, slack = _par.mfma_model(a, sa, oracle.BLOCK_1x128, b, sb, oracle.BLOCK_1x128)
    got = pre.float().cpu().numpy()[np.ix_(rows, n)]
    ratio = _par.window_check(got, model, absum, slack, "promote", K)
    print("  pre: |C - model| / bound %.3f" % ratio, flush=True)
    assert ratio <= 1.0
    acc = _par.fp32_rounding_factor("promote", K) * absum + slack
    m, e = torch.from_numpy(model), torch.from_numpy(acc)
    c = len(cols)
    g, u, dg, du = m[:, :c], m[:, c:], e[:, :c], e[:, c:]
    s = 1.0 / (1.0 + torch.exp(-g))
    ref = g * s * u
    # |silu'| <= 1.1
    lost = 1.1 * dg * (u.abs() + du) + (silu(g).abs() + 1.1 * dg) * du + 2.0 ** -18 * (ref.abs() + 1.1 * dg * u.abs())
    bound = lost + bf16_half(ref.abs() + lost)
    hs = h.float().cpu()[torch.from_numpy(rows)][:, torch.from_numpy(cols)]
    within(hs, ref, bound + 1e-40, "H")
    # without keeping: the same H; the same on every run
    same(fp8q.gemm_gated(A, sA, B, sB)[0], h, "H without pre")
    # in 8 bits: the quantization of that H
    codes, scales, pre2 = fp8q.gemm_gated_quantized(A, sA, B, sB, save=True)
    qc, qs = fp8q.quantize(h, B1)
    same(codes, qc, "codes")
    same(scales, qs, "scales")
    same(pre2, pre, "pre of the quantized call")
    again = fp8q.gemm_gated_quantized(A, sA, B, sB)
    assert again[2] is None
    same(again[0], codes, "codes of two runs")


@pytest.mark.parametrize("shape", list(ROUTES))
def test_exact_products(shape):
    """Codes of small powers of two with power-of-two scales: every product and
    sum is exact in any order, so the kept pre-activations are known bit for bit
    (a row, column or block out of place shows), and H to 2^-18 and its rounding."""
    M, K, F = shape
    g = torch.Generator().manual_seed(905)
    lut = torch.tensor([0x00, 0x38, 0xb8, 0x30, 0xb0], dtype=torch.uint8)  # 0, +-1, +-0.5
    A = lut[torch.randint(0, 5, (M, K), generator=g)]
    B = lut[torch.randint(0, 5, (2 * F, K), generator=g)]
    sA = torch.exp2(-torch.randint(3, 6, (K // 128, M), generator=g).float())
    sB = torch.exp2(-torch.randint(0, 3, (2 * F // 128, K // 128), generator=g).float())
    h, pre = fp8q.gemm_gated(A.to(DEV), sA.view(-1).to(DEV), B.to(DEV), sB.view(-1).to(DEV), save=True)
    rows = torch.unique(torch.cat((torch.arange(0, M, 1 + M // 200), torch.tensor([M - 1]))))
    a = values(A[rows]) * sA[:, rows].t().to(F64).repeat_interleave(128, dim=1)
    b = values(B) * sB.to(F64).repeat_interleave(128, 0).repeat_interleave(128, 1)
    z = (a.to(DEV) @ b.t().to(DEV)).cpu()
    same(pre.cpu()[rows], z.float().bfloat16(), "pre")
    ref = silu(z[:, :F]) * z[:, F:]
    lost = 2.0 ** -18 * ref.abs()
    within(h.cpu()[rows], ref, lost + bf16_half(ref.abs() + lost) + 1e-40, "H")


@pytest.mark.parametrize("shape", [(8, 256, 384), (300, 640, 6528), (200, 640, 16512), (2500, 1152, 8192)])
def test_strides_outputs_streams(shape):
    """Operands and outputs in wider buffers (rows of the outputs 8 bytes apart
    from 16-byte alignment too, their padding untouched), a given workspace, a
    stream of its own."""
    M, K, F = shape
    A, sA, B, sB = operands(M, K, F, seed=911)
    h, pre = fp8q.gemm_gated(A, sA, B, sB, save=True)
    codes, scales, _ = fp8q.gemm_gated_quantized(A, sA, B, sB)
    A2, B2 = strided(A, 48), strided(B, 16)
    for pad in (4, 8):
        ho = torch.full((M, F + pad), 7.0, dtype=torch.bfloat16, device=DEV)
        po = torch.full((M, 2 * F + pad), 7.0, dtype=torch.bfloat16, device=DEV)
        qo = torch.full((M, F + 16), 0xAB, dtype=torch.uint8, device=DEV)
        ws = torch.full((max(16, fp8q.lib().fp8q_gemm_gated_workspace(M, F, K)),), 0xff, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            fp8q.gemm_gated(A2, sA, B2, sB, out=ho[:, :F], pre=po[:, :2 * F])
            _, sc, _ = fp8q.gemm_gated_quantized(A2, sA, B2, sB, codes=qo[:, :F], workspace=ws)
        torch.cuda.synchronize()
        same(ho[:, :F], h, "H")
        same(po[:, :2 * F], pre, "pre")
        same(qo[:, :F], codes, "codes")
        same(sc, scales, "scales")
        assert bool((ho[:, F:] == 7).all()) and bool((po[:, 2 * F:] == 7).all()) and bool((qo[:, F:] == 0xAB).all())


def test_extreme_gates():
    """Gates of +-500 and past fp32's exp: H is the gate times up, or zero, never
    NaN."""
    M, K, F = 40, 128, 128
    A = torch.zeros(M, K, dtype=torch.uint8)
    A[:, 0] = 0x38  # 1
    B = torch.zeros(2 * F, K, dtype=torch.uint8)
    B[:F, 0] = torch.where(torch.arange(F) % 2 == 0, 0x38, 0xb8).to(torch.uint8)
    B[F:, 0] = 0x40  # 2
    sA = torch.logspace(-3, 30, M)
    h, pre = fp8q.gemm_gated(A.to(DEV), sA.to(DEV), B.to(DEV), torch.ones(2, device=DEV), save=True)
    z = sA.to(F64)[:, None] * torch.where(torch.arange(F) % 2 == 0, 1.0, -1.0).to(F64)
    ref = z / (1 + torch.exp(-z)) * 2 * sA.to(F64)[:, None]
    keep = ref.abs() < 3e38
    got = h.cpu().to(F64)
    assert not bool(torch.isnan(got).any()) and not bool(torch.isnan(pre).any())
    # (below e^-88 the exponent is held: |H| is then below 1e-36 |g u|)
    bound = bf16_half(ref * (1 + 2.0 ** -16)) + 2.0 ** -16 * ref.abs() + 1e-36 * (z * 2 * sA.to(F64)[:, None]).abs() + 1e-38
    assert bool(((got - ref).abs() <= bound)[keep].all())


def test_gated_refusals():
    A, sA, B, sB = operands(64, 256, 256, seed=915)
    f, q = fp8q.gemm_gated, fp8q.gemm_gated_quantized
    for bad in (lambda: f(A, sA[:10], B, sB), lambda: f(A, sA, B[:, :128], sB), lambda: f(A.float(), sA, B, sB),
                lambda: f(A, sA, B, sB, out=torch.empty(64, 512, dtype=torch.bfloat16, device=DEV)),
                lambda: f(A, sA, B, sB, pre=torch.empty(64, 256, dtype=torch.bfloat16, device=DEV)),
                lambda: q(A, sA, B, sB, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)),
                lambda: f(A.cpu(), sA, B, sB)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(fp8q.Fp8qError) as e:
        f(A, sA, B[:384], sB)  # F = 192: no whole blocks
    assert e.value.status == -2
    out = torch.empty(64, 258, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(fp8q.Fp8qError) as e:
        f(A, sA, B, sB, out=out[:, :256])  # ld % 4
    assert e.value.status == -3


# ---- backward

def grads(pre, dh):
    F = dh.shape[1]
    g, u, d = pre[:, :F].to(F64), pre[:, F:].to(F64), dh.to(F64)
    s = torch.sigmoid(g)
    return torch.cat((d * u * s * (1 + g * (1 - s)), d * g * s), dim=1)


def backward_inputs(M, F, seed, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    pre = (sigma * torch.randn(M, 2 * F, generator=g)).bfloat16()
    return pre, (1e-3 * torch.randn(M, F, generator=g)).bfloat16()


def check_backward(pre, dh, e5m2=False, pow2=False, out=None, rel=2.0 ** -18, tiny=0.0):
    """rel: |g| 2^-24 for the exponential (|g| up to 40) and a few roundings; near
    the root of the derivative (g = -1.28) 1 + g (1 - s) cancels, where the bound is
    of its terms, so those elements are checked with a wider one."""
    M, F = dh.shape
    cr, sr, ct, st = out or fp8q.gated_backward(dh.to(DEV), pre.to(DEV), e5m2=e5m2, pow2=pow2)
    Mp = (M + 127) // 128 * 128
    assert tuple(ct.shape) == (2 * F, Mp)
    v = grads(pre, dh)
    g = pre[:, :F].to(F64)
    s = torch.sigmoid(g)
    cancel = ((1 + g * (1 - s)).abs() < 0.05).repeat(1, 2)
    cancel[:, F:] = False
    # the cancelling elements are far below their units' maxima: hold them to the code step instead
    sc = block_scales(sr, M, 2 * F)
    assert bool(((values(cr, e5m2) * sc - v).abs()[cancel] <= sc[cancel] * 2.0 ** -6 + 0.13 * v.abs()[cancel]).all())
    vr = torch.where(cancel, values(cr, e5m2) * sc, v)
    check_units(cr, sc, vr, rel, e5m2=e5m2, pow2=pow2, tiny=tiny)
    sct = st.cpu().to(F64).view(Mp // 128, 2 * F).t().repeat_interleave(128, dim=1)
    vt = torch.zeros(2 * F, Mp, dtype=F64)
    vt[:, :M] = v.t()
    ct_cancel = torch.zeros(2 * F, Mp, dtype=torch.bool)
    ct_cancel[:, :M] = cancel.t()
    vt = torch.where(ct_cancel, values(ct, e5m2) * sct, vt)
    check_units(ct, sct, vt, rel, e5m2=e5m2, pow2=pow2, tiny=tiny)
    assert not (ct.cpu()[:, M:] & 0x7f).any()


@pytest.mark.parametrize("e5m2,pow2", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("shape", [(1, 128), (127, 128), (128, 384), (129, 256), (300, 640)])
def test_backward(shape, e5m2, pow2):
    print("gated backward", shape, e5m2, pow2, flush=True)
    check_backward(*backward_inputs(*shape, seed=921), e5m2=e5m2, pow2=pow2)


def test_backward_extremes():
    """Gates far out (s of 0 and 1, past exp's range), zeros of either sign, zero
    rows and columns, gradients so small that scales fall below 2^-90."""
    pre, dh = backward_inputs(256, 256, seed=922)
    pre[0, :256] = 3e38
    pre[1, :256] = -3e38
    pre[2, :256] = -100.0
    pre[3] = 0.0
    pre[4] = -0.0
    dh[5] = 0.0
    dh[:128, 7] = 0.0
    dh[64:70] = (dh[64:70].float() * 2.0 ** -100).bfloat16()
    pre[0, 256:] = 1.0
    pre[1, 256:] = 1.0
    out = fp8q.gated_backward(dh.to(DEV), pre.to(DEV))
    for t in (out[1], out[3]):
        assert bool(torch.isfinite(t).all())
    v = grads(pre, dh)
    sc = block_scales(out[1], 256, 512)
    got = values(out[0]) * sc
    assert bool(torch.isfinite(got).all())
    # half a code step of every element: 1/16 of it or of the smallest normal code, 2^-6, times S; rows 1 and 2: true
    # values below 1e-36 of dh g u, held to that
    big = torch.cat((dh.to(F64) * pre[:, :256].to(F64).clamp(-1e3, 1e3) * pre[:, 256:].to(F64), dh.to(F64)), dim=1).abs()
    assert bool(((got - v).abs() <= 0.0626 * v.abs() + 2.0 ** -10 * sc + 1e-35 * big).all())
    assert not (out[0].cpu()[5] & 0x7f).any()


def test_backward_against_differences():
    """sum(D t) against central differences of sum(dH H(pre)) in 64 bits along t:
    the codes' rounding is at most 1/16 of each term or 2^-10 of its scale."""
    pre, dh = backward_inputs(64, 128, seed=923)
    cr, sr, _, _ = fp8q.gated_backward(dh.to(DEV), pre.to(DEV))
    d = values(cr) * block_scales(sr, 64, 256)
    t = torch.randn(64, 256, generator=torch.Generator().manual_seed(924), dtype=F64)

    def loss(p):
        return (dh.to(F64) * silu(p[:, :128]) * p[:, 128:]).sum()

    e = 1e-5
    along = float((loss(pre.to(F64) + e * t) - loss(pre.to(F64) - e * t)) / (2 * e))
    bound = float((t.abs() * (0.0626 * d.abs() + 2.0 ** -10 * block_scales(sr, 64, 256))).sum())
    # independent roundings: their sum stays far below the sum of the bounds (4 standard deviations of it)
    spread = float((t * (0.0626 * d.abs() + 2.0 ** -10 * block_scales(sr, 64, 256))).pow(2).sum().sqrt())
    assert abs(float((d * t).sum()) - along) <= min(bound, 4 * spread) + 1e-9


def test_backward_strides_streams_far_rows():
    pre, dh = backward_inputs(200, 256, seed=925)
    want = fp8q.gated_backward(dh.to(DEV), pre.to(DEV))
    ld = 1 << 23
    far = torch.empty(200 * ld, dtype=torch.bfloat16, device=DEV).view(200, ld)[:, :512]
    far.copy_(pre)
    cr = torch.full((200, 544), 0xAB, dtype=torch.uint8, device=DEV)
    ct = torch.full((512, 272), 0xAB, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = fp8q.gated_backward(strided(dh.to(DEV), 8), far, codes_r=cr[:, :512], codes_t=ct[:, :256])
    torch.cuda.synchronize()
    for a, b, n in zip(got, want, ("codes", "scales", "transposed codes", "transposed scales")):
        same(a, b, n)
    assert bool((cr[:, 512:] == 0xAB).all()) and bool((ct[:, 256:] == 0xAB).all())


def test_backward_refusals():
    pre, dh = (t.to(DEV) for t in backward_inputs(64, 256, seed=926))
    f = fp8q.gated_backward
    for bad in (lambda: f(dh, pre[:, :256]), lambda: f(dh.float(), pre), lambda: f(dh, pre[:32]),
                lambda: f(dh, pre, codes_t=torch.empty(512, 64, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(fp8q.Fp8qError) as e:
        f(dh[:, :192], pre[:, :384])
    assert e.value.status == -2
    with pytest.raises(fp8q.Fp8qError) as e:
        f(strided(dh, 4), pre)
    assert e.value.status == -3
