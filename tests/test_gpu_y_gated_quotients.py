"""The codes of a gated activation's gradient are those of Eq. 3: the nearest to RN32(x / S),
ties to even."""
import numpy as np
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("along", ["rows", "columns"])
@pytest.mark.parametrize("e5m2", [False, True])
def test_quotients_on_the_middle_between_codes(e5m2, along):
    """Gates of zero make D = [dH U / 2 | 0] exact.  With dH = k by unit and U / 2 = m, F_max in
    every unit, S is k exactly and every x / S is m: the middles between
    codes, which go to the even one."""
    top, f8 = (57344.0, torch.float8_e5m2) if e5m2 else (448.0, torch.float8_e4m3fn)
    M = F = 256
    rng = np.random.default_rng(83)
    # middles of normal codes: 1 + (2 i + 1) / 2^(bits + 1)
    steps = 8 if e5m2 else 16
    m = (1 + np.arange(1, steps, 2) / steps)
    m = np.concatenate([m * 2.0 ** e for e in range(-4, 7)])
    m = rng.choice(np.concatenate((m, -m)), (M, F))
    m[::32, :] = top if along == "columns" else m[::32, :]
    m[:, ::32] = top if along == "rows" else m[:, ::32]
    k = rng.integers(64, 128, M) * 2 + 1
    dh = np.repeat(k[:, None], F, axis=1) if along == "rows" else np.repeat(k[None, :], M, axis=0)
    pre = np.concatenate((np.zeros((M, F)), 2 * m), axis=1)
    d, p = torch.from_numpy(dh * 2.0 ** -20).bfloat16(), torch.from_numpy(pre).bfloat16()
    assert bool((p.double().numpy() == pre).all() and (d.double().numpy() == dh * 2.0 ** -20).all())
    cr, _, ct, _ = fp8q.gated_backward(d.to(DEV), p.to(DEV), e5m2=e5m2)
    want = torch.from_numpy(np.clip(m, -top, top)).float().to(f8).view(torch.uint8)
    got = cr.cpu()[:, :F] if along == "rows" else ct.cpu()[:F, :M].t()
    assert torch.equal(got, want), int((got != want).sum())
