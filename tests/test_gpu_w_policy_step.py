"""The operators together: one FP8 policy step (examples/policy_step.py), its loss
and every gradient against the same network in 64 bits.

FP8 operands stand for their values to 2^-4 of each element (E4M3), about 2.6% of
their norm; a gradient that passed five GEMMs of two such operands each has
rounding noise of at most sqrt(10) x 2.6% = 8% and, with the forward pass's own
noise in what it is taken of, twice that: cosines of 0.97 and more."""
import importlib.util
import os

import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def exact(weights, x, branch, tokens, logp_old, adv, weight, clip, beta, logp_ref):
    w = {n: v.to(F64).requires_grad_() for n, v in weights.items()}

    def norm(h, g):
        return h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * g

    s = (x.to(F64) + branch.to(F64)).requires_grad_()
    ffn = w["up"].shape[0] // 2
    z = norm(s, w["norm"]) @ w["up"].t()
    f = z[:, :ffn] * torch.sigmoid(z[:, :ffn]) * z[:, ffn:]
    h2 = s + f @ w["down"].t()
    lp = torch.log_softmax(norm(h2, w["final"]) @ w["head"].t(), dim=1).gather(1, tokens[:, None])[:, 0]
    r, d = torch.exp(lp - logp_old.to(F64)), logp_ref.to(F64) - lp
    term = -torch.minimum(r * adv.to(F64), r.clamp(*clip) * adv.to(F64)) + beta * (torch.exp(d) - d - 1)
    loss = (weight.to(F64) * term).sum()
    loss.backward()
    return loss.detach(), {n: v.grad for n, v in w.items()}, s.grad, lp.detach()


@pytest.mark.parametrize("T,hidden,ffn,vocab", [(200, 256, 384, 1024), (1, 128, 128, 256), (513, 512, 1024, 4096)])
def test_step(example, T, hidden, ffn, vocab):
    print("policy step", T, hidden, ffn, vocab, flush=True)
    g = torch.Generator(device=DEV).manual_seed(61)
    weights = example.init(hidden, ffn, vocab, seed=62)
    x, branch = (torch.randn((T, hidden), generator=g, device=DEV).bfloat16() for _ in range(2))
    tokens = torch.randint(0, vocab, (T,), generator=g, device=DEV)
    adv = torch.randn(T, generator=g, device=DEV)
    weight = torch.full((T,), 1.0 / T, device=DEV)
    if T > 1:
        weight[::5] = 0.0
    old, _ = fp8q.token_logprobs(example.forward(weights, example.layout(weights), x, branch)[0], tokens)
    # ratios around 1, none so near a bound that FP8's noise decides the side
    old = old - torch.where(torch.rand(T, generator=g, device=DEV) < 0.3, 1.0, 0.0) * adv.sign()
    ref = old + 0.1 * torch.randn(T, generator=g, device=DEV)
    loss, grads, dx, logp, _ = example.step(weights, x, branch, tokens, old, adv, weight, beta=0.1, logp_ref=ref)
    elp = exact(weights, x, branch, tokens, old, adv, weight, (0.8, 1.24), 0.1, ref)[3]
    # the gradients at the ratios that the step saw: its log-probabilities carry the forward pass's noise, which
    # would scale each token's share
    el, eg, ex, _ = exact(weights, x, branch, tokens, old + (elp - logp), adv, weight, (0.8, 1.24), 0.1,
                          ref + (elp - logp))
    live = weight != 0
    # a logit is a product of two quantized operands, of standard deviation about 1: 2.6% sqrt(2) and the
    # noise of what is in front of it
    assert float((logp - elp)[live].abs().mean()) < 0.15
    for n in list(eg) + ["dx"]:
        a, b = (dx, ex) if n == "dx" else (grads[n].view(eg[n].shape), eg[n])
        a = a.to(F64)
        cos = float((a * b).sum() / (a.norm() * b.norm()))
        print("  %s: cosine %.4f, norms %.3f" % (n, cos, float(a.norm() / b.norm())), flush=True)
        assert cos > 0.97 and abs(float(a.norm() / b.norm()) - 1) < 0.1, n


def test_demo_learns(example):
    """A few steps on one batch lower its loss."""
    losses = example.demo(tokens=300, hidden=256, ffn=512, vocab=1024)
    assert losses[-1] < losses[0] - 0.1
