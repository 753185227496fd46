"""Tokens in, tokens out, and a training step on them: the policy of policy_step.py
between an embedding table and sampled alternatives, on the package's entry points.

    python examples/rollout_step.py [batch length hidden ffn vocab]

The rollout runs the gated projections in FP8 and the down and output projections in
MXFP4 (4-bit codes, a scale per 32 elements; laid out once per update), and takes each
next token among the k most probable ones.  A position sees its own token's row of the
table and, in place of an attention branch, half the previous one's.  Training runs the
same tokens through the FP8 step and adds both uses' gradients into one table's.
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2609_22870_amd as fp8q  # noqa: E402

import policy_step  # noqa: E402

B1, B128, EPS = policy_step.B1, policy_step.B128, policy_step.EPS
BRANCH = 0.5  # the previous token's share


def init(hidden, ffn, vocab, seed=0, device="cuda"):
    """policy_step's weights and the table."""
    g = torch.Generator(device=device).manual_seed(seed + 1)
    return dict(policy_step.init(hidden, ffn, vocab, seed, device),
                table=torch.randn((vocab, hidden), generator=g, device=device).bfloat16())


def layout(weights):
    """The rollout's operands, made once per update."""
    return dict(up=fp8q.quantize(weights["up"], B128), down=fp8q.quantize_mx4(weights["down"]),
                head=fp8q.quantize_mx4(weights["head"]))


def inputs(table, tokens, previous):
    """The residual stream and the branch of positions that hold `tokens`; -1: none."""
    return fp8q.embedding(table, tokens), fp8q.embedding(table, previous, BRANCH)


def logits(weights, ops, tokens, previous):
    """bf16 [T, vocab] of positions that hold `tokens`."""
    x, branch = inputs(weights["table"], tokens, previous)
    a, sa, h, _ = fp8q.rmsnorm_quantize(x, weights["norm"], EPS, residual=branch, h=x)
    f, _ = fp8q.gemm_gated(a, sa, *ops["up"])
    y = fp8q.gemm_mx4(*fp8q.quantize_mx4(f), *ops["down"])
    z, _, _ = fp8q.rmsnorm(y, weights["final"], EPS, residual=h, h=h)
    return fp8q.gemm_mx4(*fp8q.quantize_mx4(z), *ops["head"])


def generate(weights, ops, prompt, length, k=20, generator=None):
    """`length` tokens after each of prompt's [batch], and their log-probabilities:
    int64 and fp32 [batch, length]."""
    none = torch.full_like(prompt, -1)
    tokens, previous, taken, logps = prompt, none, [], []
    for _ in range(length):
        # (the token is not known yet: 0 in its place, its log-probability read from the alternatives)
        _, _, ids, top = fp8q.top_logprobs(logits(weights, ops, tokens, previous), torch.zeros_like(tokens), k)
        i = torch.multinomial(top.exp(), 1, generator=generator)
        tokens, previous = ids.gather(1, i)[:, 0], tokens
        taken.append(tokens)
        logps.append(top.gather(1, i)[:, 0])
    return torch.stack(taken, 1), torch.stack(logps, 1)


def positions(prompt, taken):
    """(tokens, previous, next) of every position that led to one of `taken`, one sequence
    after the other."""
    seq = torch.cat((torch.full_like(prompt, -1)[:, None], prompt[:, None], taken), 1)
    return tuple(seq[:, i:i + taken.shape[1]].reshape(-1).contiguous() for i in (1, 0, 2))


def score(weights, ops, prompt, taken, k=20):
    """Log-probabilities, entropies and alternatives of `taken`, all positions at once."""
    tokens, previous, following = positions(prompt, taken)
    return fp8q.top_logprobs(logits(weights, ops, tokens, previous), following, k)


def step(weights, prompt, taken, logp_old, adv, weight, grad_scale=1024.0, **loss):
    """(loss, gradients, log-probabilities) of one batch of rollouts; the table's gradient
    among them, fp32 [vocab, hidden]."""
    tokens, previous, following = positions(prompt, taken)
    x, branch = inputs(weights["table"], tokens, previous)
    policy = {n: w for n, w in weights.items() if n != "table"}
    total, grads, dx, logp, _ = policy_step.step(policy, x, branch, following, logp_old.reshape(-1), adv, weight,
                                                 grad_scale=grad_scale, **loss)
    d = (dx * grad_scale).bfloat16()  # (as the step made it: a power of two)
    vocab = weights["table"].shape[0]
    table = fp8q.embedding_backward(d, tokens, vocab, 1.0 / grad_scale)
    grads["table"] = fp8q.embedding_backward(d, previous, vocab, BRANCH / grad_scale, dweight=table, accumulate=True)
    return total, grads, logp


def demo(batch=16, length=32, hidden=1024, ffn=2048, vocab=8192):
    g = torch.Generator(device="cuda").manual_seed(2)
    weights = init(hidden, ffn, vocab)
    ops = layout(weights)
    prompt = torch.randint(0, vocab, (batch,), generator=g, device="cuda")
    taken, logp_old = generate(weights, ops, prompt, length, generator=g)
    logp, entropy, ids, top = score(weights, ops, prompt, taken)
    print("%d tokens: mean log-probability %.3f, entropy %.3f, the 20 alternatives' share %.3f" % (
        taken.numel(), float(logp.mean()), float(entropy.mean()), float(top.exp().sum(1).mean())), flush=True)
    adv = torch.randn(taken.numel(), generator=g, device="cuda")
    weight = torch.full((taken.numel(),), 1.0 / taken.numel(), device="cuda")
    loss, grads, _ = step(weights, prompt, taken, logp_old, adv, weight)
    print("loss %.5f, gradient norms %s" % (float(loss), {n: "%.2e" % float(v.norm()) for n, v in grads.items()}), flush=True)
    return loss, grads


if __name__ == "__main__":
    demo(*(int(a) for a in sys.argv[1:6]))
