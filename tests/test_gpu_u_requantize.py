"""Activations kept in 8 bits as weight-gradient operands: the transposed codes
in units of 128 rows against the definition, v = fp32(S code), S' =
fp32(amax / 448), codes of v / S'.

v and S' are single correctly rounded operations, the same in the reference:
scales must match bit for bit, and a code may differ from the nearest one only
where v / S' lies within 2^-22 of the middle between two codes."""
import numpy as np
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, block_scales, check_units, same, values

pytestmark = pytest.mark.gpu


def kept(rows, cols, seed, gain=None):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    x[:, ::41] *= 50.0
    if gain is not None:
        x *= gain
    return fp8q.quantize(x.bfloat16().to(DEV), fp8q.BLOCK_1x128)


def check(codes, scales, out, rows, cols, pow2=False):
    ct, st = out
    Rp = (rows + 127) // 128 * 128
    v = (values(codes).float() * block_scales(scales, rows, cols).float()).to(F64)  # one fp32 product
    v = torch.cat((v, torch.zeros(Rp - rows, cols, dtype=F64)))
    assert tuple(ct.shape) == (cols, Rp) and st.numel() == Rp // 128 * cols
    s = st.cpu().view(Rp // 128, cols)
    if not pow2:
        amax = v.abs().view(-1, 128, cols).amax(dim=1).float()
        want = amax / np.float32(448.0)
        want = torch.where(want == 0, torch.ones_like(want), want)
        assert torch.equal(s, want), "scales"
    assert not (ct.cpu()[:, rows:] & 0x7f).any(), "padding"
    check_units(ct, s.t().to(F64).repeat_interleave(128, dim=1), v.t().contiguous(), 0.0, pow2=pow2)


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("shape", [(1, 128), (127, 256), (128, 384), (129, 128), (300, 1280), (1001, 5120)])
def test_against_definition(shape, pow2):
    print("requantize", shape, pow2, flush=True)
    codes, scales = kept(*shape, seed=21)
    check(codes, scales, fp8q.requantize_transposed(codes, scales, pow2=pow2), *shape, pow2=pow2)


def test_every_code_and_special_units():
    """Every finite code in a unit of its own scale, columns of zeros, and scales
    down to fp32's subnormals (products and S' below 2^-90, S' of 0)."""
    rows, cols = 256, 256
    codes = torch.arange(256, dtype=torch.uint8).repeat(rows // 256 * cols).view(cols, rows).t().contiguous()
    codes[(codes & 0x7f) == 0x7f] = 0x3a  # NaN codes are outside the contract
    codes[:, 5] = 0x80
    codes[:128, 6] = 0
    scales = torch.ones(cols // 128, rows)
    scales[0] = torch.exp2(torch.linspace(-40, 40, rows))
    scales[1, :128] = 2.0 ** -141
    scales[1, 128:] = 2.0 ** -96
    codes, scales = codes.to(DEV), scales.view(-1).to(DEV)
    out = fp8q.requantize_transposed(codes, scales)
    ct, st = out
    v = (values(codes).float() * block_scales(scales, rows, cols).float())
    amax = v.abs().view(2, 128, cols).amax(dim=1)
    want = amax / np.float32(448.0)
    want = torch.where(want == 0, torch.ones_like(want), want)
    assert torch.equal(st.cpu().view(2, cols), want)
    s = want.t().to(F64).repeat_interleave(128, dim=1)
    keep = [c for c in range(cols)]
    check_units(ct[keep], s[keep], v.t().to(F64).contiguous()[keep], 0.0, tiny=2.0 ** -149)


def test_strides_given_outputs_and_far_rows():
    """Rows that start past 2^31 bytes, wide outputs (their padding untouched), on
    a stream of its own."""
    rows, cols, ld = 300, 256, 1 << 23
    codes, scales = kept(rows, cols, seed=22)
    want = fp8q.requantize_transposed(codes, scales)
    far = torch.empty(rows * ld, dtype=torch.uint8, device=DEV).view(rows, ld)[:, :cols]
    far.copy_(codes)
    wide = torch.full((cols, 416), 0xAB, dtype=torch.uint8, device=DEV)
    st = torch.empty(3 * cols, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = fp8q.requantize_transposed(far, scales, codes_t=wide[:, :384], scales_t=st)
    torch.cuda.synchronize()
    same(got[0], want[0], "codes")
    same(got[1], want[1], "scales")
    assert bool((wide[:, 384:] == 0xAB).all())


def test_feeds_the_weight_gradient():
    """dW = dY^T X with X from kept codes of a ragged number of tokens: the GEMM
    on its operand equals the product of what both operands stand for, to the
    rounding of the output and the instruction's truncation (5e-3 of the row)."""
    rows, cols, n = 333, 256, 128
    codes, scales = kept(rows, cols, seed=23)
    xt, sxt = fp8q.requantize_transposed(codes, scales)
    dy = torch.zeros(384, n, dtype=torch.bfloat16)
    dy[:rows] = (torch.randn(rows, n, generator=torch.Generator().manual_seed(24)) * 1e-3).bfloat16()
    dt, sdt = fp8q.quantize(dy.to(DEV), fp8q.BLOCK_128x1, transposed=True)
    dw = fp8q.gemm(dt, sdt, fp8q.BLOCK_1x128, xt, sxt, fp8q.BLOCK_1x128).cpu().to(F64)
    a = values(dt) * sdt.cpu().to(F64).view(3, n).t().repeat_interleave(128, dim=1)
    b = values(xt) * sxt.cpu().to(F64).view(3, cols).t().repeat_interleave(128, dim=1)
    ref = a @ b.t()
    assert bool(((dw - ref).abs() <= 5e-3 * ref.abs().amax(dim=1, keepdim=True)).all())


def test_refusals():
    codes, scales = kept(128, 256, seed=25)
    call = fp8q.requantize_transposed
    for bad in (lambda: call(codes.float(), scales), lambda: call(codes, scales[:100]),
                lambda: call(codes, scales, codes_t=torch.empty(256, 100, dtype=torch.uint8, device=DEV)),
                lambda: call(codes.cpu(), scales), lambda: call(codes, scales.cpu())):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros(128, 400, dtype=torch.uint8, device=DEV)
    with pytest.raises(fp8q.Fp8qError) as e:
        call(odd[:, :200], torch.zeros(400, device=DEV))
    assert e.value.status == -2
    with pytest.raises(fp8q.Fp8qError) as e:
        call(odd[:, 1:257], torch.zeros(400, device=DEV))
    assert e.value.status == -3
