"""What the gated activation loses before its last rounding, at gates far from zero, where exp(-g)
from one rounded product would be off by |g| 2^-24 of itself.

The bound, in units of 2^-24 of the value: v_exp_f32 and v_rcp_f32 are good to an ulp
(2), a product, a sum or a fused multiply-add to half of one (1), and what ln 2 in
fp32 leaves of the exponent's correction is |g| 2.8e-9 (4 at |g| = 86).  silu(g) u takes exp,
the correction's sum and product, 1 + e, the reciprocal and two products: 13 in all, below
2^-20."""
import numpy as np
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, bf16_half, gated_route, values, within

pytestmark = pytest.mark.gpu


# (a kernel of every form of the epilogue)
@pytest.mark.parametrize("shape", [(8, 1152, 1024), (61, 256, 8192), (300, 128, 1152), (300, 640, 6528), (200, 640, 16512)])
def test_forward(shape):
    """Products exact in any order, gates -86 .. 86 of some 20 bits: H is silu(g) u to 2^-20 and its
    last rounding."""
    M, K, F = shape
    print("gated precision", shape, gated_route(M, F, K), flush=True)
    rng = np.random.default_rng(81)
    # row m: 1 and 1/8; gate f: the same of two codes of 1 .. 16
    lut = torch.arange(128, dtype=torch.uint8)
    lut = lut[(values(lut) >= 1) & (values(lut) <= 16)]
    A = torch.zeros(M, K, dtype=torch.uint8)
    A[:, 0], A[:, 1] = 0x38, 0x20  # 1, 1/8
    B = torch.zeros(2 * F, K, dtype=torch.uint8)
    B[:F, 0] = torch.from_numpy(rng.choice(lut.numpy(), F))
    B[:F, 1] = torch.from_numpy(rng.choice(lut.numpy(), F))
    B[F:, 0] = 0x38
    sA = torch.zeros(K // 128, M)
    # the row's scale, of 12 bits, so that every |gate| is below 86
    sA[0] = torch.from_numpy(np.sign(rng.random(M) - 0.25) * rng.integers(1024, 2458, M) / 1024.0 * 2.0).float()
    sA[1:] = 1.0
    sB = torch.ones(2 * F // 128, K // 128)
    h, _ = fp8q.gemm_gated(A.to(DEV), sA.view(-1).to(DEV), B.to(DEV), sB.view(-1).to(DEV))
    g = (values(B[:F, 0]) + values(B[:F, 1]) / 8)[None, :] * sA[0].to(F64)[:, None]
    u = sA[0].to(F64)[:, None].expand(M, F)
    # (the GEMM's fp32 sum is the gate exactly: 11 bits of codes times 12 of the scale)
    assert torch.equal(g.float().to(F64), g)
    ref = g / (1 + torch.exp(-g)) * u
    keep = g.abs() < 86
    assert float(keep.to(F64).mean()) > 0.9 and float(g[keep].min()) < -50
    lost = 2.0 ** -20 * ref.abs()
    within(h.cpu()[keep], ref[keep], (lost + bf16_half(ref.abs() + lost))[keep], "H")
