"""One training step of a small FP8 policy: a norm, a gated feed-forward block on
the residual stream, a final norm and the output projection, and the clipped policy
loss, forward and backward, on the package's entry points.

    python examples/policy_step.py [tokens hidden ffn vocab]

The linear layers run in FP8 (activations and gradients per 1x128 block, weights
per 128x128 block).  What the forward pass keeps for the backward pass is the
residual stream in bf16 with each norm's rstd, the gate's and up projection's
outputs, and the FP8 codes that the GEMMs took: their transposes for the weight
gradients are requantized from those codes.  Token counts need not be multiples
of 128; the hidden, FFN and vocabulary sizes do.
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_22870_amd as fp8q  # noqa: E402

B1, B128 = fp8q.BLOCK_1x128, fp8q.BLOCK_128x128
EPS = 1e-6


def init(hidden, ffn, vocab, seed=0, device="cuda"):
    """bf16 weights: two norms, gate and up projections one below the other, down
    projection, output projection."""
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, sigma):
        return torch.randn(shape, generator=g, device=device).mul_(sigma).bfloat16()

    return dict(norm=torch.ones(hidden, device=device).bfloat16(), up=normal(2 * ffn, hidden, sigma=hidden ** -0.5),
                down=normal(hidden, ffn, sigma=ffn ** -0.5), final=torch.ones(hidden, device=device).bfloat16(),
                head=normal(vocab, hidden, sigma=hidden ** -0.5))


def layout(weights):
    """The weights' FP8 operands, made once per update: each projection's for the
    forward GEMM and, transposed, for the data gradient's."""
    return {n: (fp8q.quantize(w, B128), fp8q.quantize(w, B128, transposed=True))
            for n, w in weights.items() if w.dim() == 2}


def forward(weights, ops, x, branch):
    """Logits for the residual stream x and the attention branch's output (added to
    it first); and what backward() needs."""
    k = {}
    k["a"], k["sa"], k["h"], k["rstd"] = fp8q.rmsnorm_quantize(x, weights["norm"], EPS, residual=branch)
    k["f"], k["sf"], k["pre"] = fp8q.gemm_gated_quantized(k["a"], k["sa"], *ops["up"][0], save=True)
    y = fp8q.gemm(k["f"], k["sf"], B1, *ops["down"][0], B128)
    k["z"], k["sz"], k["h2"], k["rstd2"] = fp8q.rmsnorm_quantize(y, weights["final"], EPS, residual=k["h"])
    return fp8q.gemm(k["z"], k["sz"], B1, *ops["head"][0], B128), k


def _both(d):
    """A gradient's operands: per 1x128 block, and transposed in units of 128
    tokens (rows of zeros fill the last one up)."""
    pad = -d.shape[0] % 128
    if not pad:
        return fp8q.quantize_dual(d)
    codes_t, scales_t = fp8q.quantize(torch.nn.functional.pad(d, (0, 0, 0, pad)), fp8q.BLOCK_128x1, transposed=True)
    return fp8q.quantize(d, B1) + (codes_t, scales_t)


def _weight_gradient(codes_t, scales_t, kept, kept_scales):
    """dW = dY^T X from dY's transposed codes and the codes X was kept in."""
    xt, sxt = fp8q.requantize_transposed(kept, kept_scales)
    return fp8q.gemm(codes_t, scales_t, B1, xt, sxt, B1)


def backward(weights, ops, k, dlogits):
    """Gradients of the weights, and of the residual stream (and of the branch: the
    same)."""
    g = {}
    d, sd, dt, sdt = _both(dlogits)
    g["head"] = _weight_gradient(dt, sdt, k["z"], k["sz"])
    dz = fp8q.gemm(d, sd, B1, *ops["head"][1], B128)
    dh2, g["final"] = fp8q.rmsnorm_backward(dz, k["h2"], k["rstd2"], weights["final"])
    d, sd, dt, sdt = _both(dh2)
    g["down"] = _weight_gradient(dt, sdt, k["f"], k["sf"])
    df = fp8q.gemm(d, sd, B1, *ops["down"][1], B128)
    d, sd, dt, sdt = fp8q.gated_backward(df, k["pre"])
    g["up"] = _weight_gradient(dt, sdt, k["a"], k["sa"])
    da = fp8q.gemm(d, sd, B1, *ops["up"][1], B128)
    dx, g["norm"] = fp8q.rmsnorm_backward(da, k["h"], k["rstd"], weights["norm"], dres=dh2)
    return g, dx


def step(weights, x, branch, tokens, logp_old, adv, weight, clip=(0.8, 1.24), beta=0.0, logp_ref=None, grad_scale=1024.0):
    """(loss, gradients, dx, log-probabilities, entropies) of one batch.  The
    gradient is taken of grad_scale times the loss, so that its bf16 values keep
    their bits, and divided again."""
    ops = layout(weights)
    logits, k = forward(weights, ops, x, branch)
    loss, dlogits, logp, entropy = fp8q.policy_loss(logits, tokens, logp_old, adv, weight * grad_scale, *clip, beta=beta,
                                                    logp_ref=logp_ref, dlogits=logits)
    grads, dx = backward(weights, ops, k, dlogits)
    return loss / grad_scale, {n: v.float() / grad_scale for n, v in grads.items()}, dx.float() / grad_scale, logp, entropy


def demo(tokens=1000, hidden=1024, ffn=2048, vocab=8192, steps=6, rate=0.002):
    g = torch.Generator(device="cuda").manual_seed(1)
    weights = init(hidden, ffn, vocab)
    x, branch = (torch.randn((tokens, hidden), generator=g, device="cuda").bfloat16() for _ in range(2))
    taken = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    adv = torch.randn(tokens, generator=g, device="cuda")
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    losses = []
    logp_old, _ = fp8q.token_logprobs(forward(weights, layout(weights), x, branch)[0], taken)
    for i in range(steps):
        loss, grads, _, logp, entropy = step(weights, x, branch, taken, logp_old, adv, weight, beta=0.01, logp_ref=logp_old)
        losses.append(float(loss))
        print("step %d: loss %.5f, entropy %.3f, mean ratio of A > 0 %.3f, of A < 0 %.3f" % (
            i, losses[-1], float(entropy.mean()), float((logp - logp_old).exp()[adv > 0].mean()),
            float((logp - logp_old).exp()[adv < 0].mean())), flush=True)
        for n, d in grads.items():
            w = weights[n].float()  # (a step of `rate` of the weight's norm along its gradient)
            weights[n] = (w - rate * w.norm() / d.norm().clamp(min=1e-20) * d.view_as(w)).bfloat16()
    return losses


if __name__ == "__main__":
    demo(*(int(a) for a in sys.argv[1:5]))
