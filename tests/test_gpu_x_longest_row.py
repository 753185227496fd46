"""The longest row of logits that the calls take, 2^31 - 1 of them: the elements before and
after its whole 16-byte pieces count, and get their gradients.

Every logit is 0 but the first and the last few, which hold most of the probability
between them, so that one left out shows at once.  Sums of ones are exact in fp32 up
to 2^24 a thread; 2^-18 of the logarithm has room for the exponentials and the joins."""
import math

import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV

pytestmark = pytest.mark.gpu

V = 2 ** 31 - 1


@pytest.mark.parametrize("start", [0, 1])  # (a row on a 16-byte boundary, and one off it)
def test_longest_row(start):
    print("longest row, start", start, flush=True)
    buffer = torch.zeros(V + 8, dtype=torch.bfloat16, device=DEV)
    x = buffer[start:start + V].view(1, V)
    x[0, :3] = 24.0
    x[0, -3:] = 24.0
    lse = math.log(V - 6 + 6 * math.exp(24.0))
    one = torch.ones(1, device=DEV)
    for token in (0, V - 1, V // 2):
        logp, entropy = fp8q.token_logprobs(x, torch.tensor([token], device=DEV))
        want = float(x[0, token]) - lse
        p = math.exp(24.0 - lse)
        assert abs(float(logp) - want) <= 2.0 ** -18 * lse, token
        assert abs(float(entropy) - (lse - 6 * p * 24.0)) <= 2.0 ** -16 * lse, token
    d = torch.full((V + 8,), 7.0, dtype=torch.bfloat16, device=DEV)
    tokens = torch.tensor([V - 1], device=DEV)
    old = torch.full((1,), 24.0 - lse, device=DEV)
    _, g, logp, _ = fp8q.policy_loss(x, tokens, old, one, one, 0.5, 2.0, dlogits=d[start:start + V].view(1, V))
    assert abs(float(logp) - (24.0 - lse)) <= 2.0 ** -18 * lse
    # ratio 1, advantage 1: the derivative in logp is -1, so the gradient is p - delta
    want = torch.full((6,), p, dtype=torch.float64)
    want[5] -= 1.0
    got = torch.cat((g[0, :3], g[0, -3:])).double().cpu()
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs()).all()), got
    rest = g[0, 3:-3]
    assert float(rest.amax()) == float(rest.amin())
    assert abs(float(rest[0]) - math.exp(-lse)) <= 2.0 ** -8 * math.exp(-lse)
    assert bool((d[:start] == 7).all()) and bool((d[start + V:] == 7).all())
