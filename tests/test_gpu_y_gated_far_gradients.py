"""What a gated activation's gradient loses before its last rounding, at gates far from zero, where
exp(-g) from one rounded product would be off by |g| 2^-24 of itself.

Bounds, in units of 2^-24 of the value: v_exp_f32 and v_rcp_f32 are good to an ulp
(2), a product, a sum or a fused multiply-add to half of one (1), and the exponent's
correction leaves 1.5 (its second order at |g| = 87).  dG = dH U s (1 + G (1 - s)) takes exp,
the correction's two, 1 + e, the reciprocal, four products, 1 - s and the factor's fused
multiply-add, whose terms cancel to no less than 1 / 1.5 of their magnitudes below G = -5: 17
at most, below 2^-19.  Above zero the rounding of s next to 1 counts G times in 1 - s (until
1 + e is 1, G = 17): 17 x 2.5 more, below 2^-18."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, block_scales, check_units

pytestmark = pytest.mark.gpu


def backward(pre, dh, rel, e5m2=False):
    M, F = dh.shape
    cr, sr, ct, st = fp8q.gated_backward(dh.to(DEV), pre.to(DEV), e5m2=e5m2)
    g, u, d = pre[:, :F].to(F64), pre[:, F:].to(F64), dh.to(F64)
    s = 1 / (1 + torch.exp(-g))
    v = torch.cat((d * u * s * (1 + g * (1 - s)), d * g * s), dim=1)
    check_units(cr, block_scales(sr, M, 2 * F), v, rel, e5m2=e5m2)
    sct = st.cpu().to(F64).view(M // 128, 2 * F).t().repeat_interleave(128, dim=1)
    check_units(ct, sct, v.t().contiguous(), rel, e5m2=e5m2)


@pytest.mark.parametrize("e5m2", [False, True])
@pytest.mark.parametrize("sign", [-1, 1])
def test_backward_far_gates(sign, e5m2):
    """Every 128 x 128 tile at a gate of its own, 5 .. 80 from zero."""
    M, F = 512, 2048
    g = torch.Generator().manual_seed(82)
    far = sign * torch.linspace(5, 80, M // 128 * F // 128).view(M // 128, F // 128)
    gate = far.repeat_interleave(128, 0).repeat_interleave(128, 1) * (1 + 0.01 * torch.rand(M, F, generator=g))
    pre = torch.cat((gate, torch.randn(M, F, generator=g)), dim=1).bfloat16()
    backward(pre, torch.randn(M, F, generator=g).bfloat16(), 2.0 ** (-19 if sign < 0 else -18), e5m2)
