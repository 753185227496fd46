"""The operators together: a rollout in 4 bits from tokens to sampled tokens, its scores,
and a training step down to the embedding table (examples/rollout_step.py), against the same
network in 64 bits; a decode step captured into a graph; calls from another stream, in inference
mode and seen by dispatch modes, as all the package's calls."""
import importlib.util
import os

import pytest
import torch

import paper_2609_22870_amd as fp8q

import _mx4
from _ops import DEV, F64, same
from test_gpu_z_allocation import Seen

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("rollout_step", os.path.join(ROOT, "examples", "rollout_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def network(w, tokens, previous):
    """Logits in 64 bits of unquantized operands."""
    def rows(t):
        return torch.where((t >= 0)[:, None], w["table"][t.clamp(min=0)], torch.zeros((), dtype=F64, device=t.device))

    def norm(h, g):
        return h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * g

    h = rows(tokens) + 0.5 * rows(previous)
    ffn = w["up"].shape[0] // 2
    z = norm(h, w["norm"]) @ w["up"].t()
    return norm(h + (torch.nn.functional.silu(z[:, :ffn]) * z[:, ffn:]) @ w["down"].t(), w["final"]) @ w["head"].t()


def cosine(a, b):
    a, b = a.to(F64).reshape(-1), b.to(F64).reshape(-1)
    return float((a * b).sum() / (a.norm() * b.norm()))


@pytest.mark.parametrize("batch,length,hidden,ffn,vocab", [(5, 9, 256, 384, 1000), (1, 1, 128, 128, 260),
                                                           (24, 16, 512, 1024, 4096)])
def test_rollout(example, batch, length, hidden, ffn, vocab):
    """Each level of E2M1 is nearer than a quarter of the value to what it stands for (at 1.25, and
    at the clamp from 8 to 6), above half the smallest; over a unit's Gaussian values the error's norm is
    at most 16% of theirs (steps of 1/2, 1 and 2 over an amax of 4 to 8: a mean square of about 0.1 of the
    scale's square, of at least 4).  Four such operands and three in FP8 (3%): 33% of a logit's norm at most, a
    cosine of 0.94 and more."""
    print("rollout", batch, length, hidden, ffn, vocab, flush=True)
    g = torch.Generator(device=DEV).manual_seed(81)
    weights = example.init(hidden, ffn, vocab, seed=82)
    ops = example.layout(weights)
    prompt = torch.randint(0, vocab, (batch,), generator=g, device=DEV)
    k = 12
    taken, logps = example.generate(weights, ops, prompt, length, k, generator=g)
    assert taken.shape == logps.shape == (batch, length) and taken.dtype == torch.int64
    assert int(taken.min()) >= 0 and int(taken.max()) < vocab and float(logps.max()) <= 0
    tokens, previous, following = example.positions(prompt, taken)
    x = example.logits(weights, ops, tokens, previous)
    logp, entropy, ids, top = fp8q.top_logprobs(x, following, k)
    # the scores, from the logits as they came out
    lp = torch.log_softmax(x.to(F64), dim=1)
    assert float((logp - lp.gather(1, following[:, None])[:, 0]).abs().max()) < 1e-4
    assert float((entropy + (lp.exp() * lp).sum(1)).abs().max()) < 1e-4
    for a, b in zip(example.score(weights, ops, prompt, taken, k), (logp, entropy, ids, top)):
        same(a, b, "score")
    # a decode step's rows, in small products, and all positions' at once: one rounding of a logit to bf16 apart
    # (its largest is below 8: 2^-6 at most) for each of the two terms of a log-probability, and what their
    # last norm's and its quantizer's ties make of one
    assert float((logps.reshape(-1) - logp).abs().mean()) < 2 * 2.0 ** -6
    w = {n: v.to(F64) for n, v in weights.items()}
    exact = network(w, tokens, previous)
    c = cosine(x, exact)
    print("  logits: cosine %.4f" % c, flush=True)
    assert c > 0.94
    # the output projection by itself, on its own operands
    z = torch.randn((batch, hidden), generator=g, device=DEV).bfloat16()
    y = fp8q.gemm_mx4(*fp8q.quantize_mx4(z), *ops["head"]).cpu().to(F64)
    va, vb = (_mx4.values(*_mx4.quantize(t.cpu())) for t in (z, weights["head"]))
    bound = 2.0 ** -8 * (va @ vb.t()).abs() + va.shape[1] * 2.0 ** -22 * (va.abs() @ vb.abs().t())
    assert bool(((y - va @ vb.t()).abs() <= bound).all())


@pytest.mark.parametrize("batch,length,hidden,ffn,vocab", [(6, 20, 256, 384, 1024), (1, 1, 128, 128, 256),
                                                           (27, 19, 512, 1024, 4096)])
def test_step(example, batch, length, hidden, ffn, vocab):
    """The table's gradient of the whole step: of its noise as the stream's gradient that it sums (see
    test_gpu_w_policy_step)."""
    print("rollout step", batch, length, hidden, ffn, vocab, flush=True)
    g = torch.Generator(device=DEV).manual_seed(83)
    weights = example.init(hidden, ffn, vocab, seed=84)
    prompt = torch.randint(0, vocab, (batch,), generator=g, device=DEV)
    taken, _ = example.generate(weights, example.layout(weights), prompt, length, 12, generator=g)
    n = taken.numel()
    adv = torch.randn(n, generator=g, device=DEV)
    weight = torch.full((n,), 1.0 / n, device=DEV)
    old = torch.zeros(n, device=DEV)
    # (no bound: the ratios of old = 0 are the tokens' probabilities)
    loss, grads, logp = example.step(weights, prompt, taken, old, adv, weight, clip=(0.0, 2.0))
    w = {m: v.to(F64).requires_grad_() for m, v in weights.items()}
    tokens, previous, following = example.positions(prompt, taken)
    lp = torch.log_softmax(network(w, tokens, previous), dim=1).gather(1, following[:, None])[:, 0]
    # (the gradients at the ratios that the step saw)
    exact = -(weight.to(F64) * adv.to(F64) * torch.exp(lp + (logp.to(F64) - lp).detach())).sum()
    exact.backward()
    assert abs(float(loss - exact.detach())) <= 1e-4 * float((weight * adv.abs() * logp.exp()).sum())
    for m, v in w.items():
        c = cosine(grads[m].view(v.shape), v.grad)
        print("  %s: cosine %.4f" % (m, c), flush=True)
        assert c > 0.97 and abs(float(grads[m].norm() / v.grad.norm()) - 1) < 0.1, m
    used = torch.zeros(vocab, dtype=torch.bool, device=DEV)
    used[tokens] = True
    used[previous[previous >= 0]] = True
    assert not bool(grads["table"][~used].any())


def test_demo(example):
    loss, grads = example.demo(batch=4, length=8, hidden=256, ffn=512, vocab=1024)
    assert bool(torch.isfinite(loss)) and all(bool(torch.isfinite(v).all()) for v in grads.values())


def test_decode_step_captured(example):
    """One step's launches in a graph, replayed with other tokens, eager work between."""
    hidden, vocab, batch, k = 256, 1000, 5, 7
    weights = example.init(hidden, 384, vocab, seed=85)
    ops = example.layout(weights)
    tokens, previous = (torch.zeros(batch, dtype=torch.int64, device=DEV) for _ in range(2))

    def run():
        return fp8q.top_logprobs(example.logits(weights, ops, tokens, previous), tokens, k)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in range(4):
        t = torch.randint(-1, vocab, (2, batch), generator=torch.Generator().manual_seed(seed)).to(DEV)
        tokens.copy_(t[0])
        previous.copy_(t[1])
        graph.replay()
        got = [o.clone() for o in out]
        for a, b in zip(got, run()):
            same(a, b, "replay %d" % seed)
        torch.cuda.synchronize()


def calls():
    g = torch.Generator().manual_seed(86)
    x = torch.randn(40, 320, generator=g).bfloat16().to(DEV)
    codes, scales = fp8q.quantize_mx4(x)
    tokens = torch.randint(-1, 40, (24,), generator=g).to(DEV)
    # (name, call, new tensors)
    return (("quantize_mx4", lambda: fp8q.quantize_mx4(x), 2), ("dequantize_mx4", lambda: fp8q.dequantize_mx4(codes, scales, 320), 1),
            ("gemm_mx4", lambda: fp8q.gemm_mx4(codes, scales, codes, scales), 1),
            ("embedding", lambda: fp8q.embedding(x, tokens), 1),
            ("embedding_backward", lambda: fp8q.embedding_backward(x[:24], tokens, 40), 2),
            # (short rows need no workspace: an empty one)
            ("top_logprobs", lambda: fp8q.top_logprobs(x[:24], tokens, 5), None))


def test_new_tensors_and_streams():
    """New tensors come from torch.empty, in the current inference mode, and the work runs on the
    current stream."""
    for name, call, new in calls():
        want = call()
        want = want if isinstance(want, tuple) else (want,)
        torch.cuda.synchronize()
        with Seen() as seen:
            got = call()
        made = sum(n.startswith("aten::empty.") for n in seen.names)
        assert made == new or (new is None and made in (4, 5)), (name, seen.names)
        stream = torch.cuda.Stream()
        with torch.inference_mode(), torch.cuda.stream(stream):
            there = call()
        stream.synchronize()
        for r in (got, there):
            for a, b in zip(r if isinstance(r, tuple) else (r,), want):
                same(a, b, name)
                assert a.is_contiguous() and a.device == b.device and a.is_inference() == (r is there)


def test_two_streams_at_once():
    """The same calls on two streams at once: nothing is shared between them."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = [(name, call, call()) for name, call, _ in calls()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append([call() for _, call, _ in want])
    torch.cuda.synchronize()
    for results in got:
        for (name, _, w), r in zip(want, results):
            for a, b in zip(r if isinstance(r, tuple) else (r,), w if isinstance(w, tuple) else (w,)):
                same(a, b, name)
