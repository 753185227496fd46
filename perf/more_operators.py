"""The operators of a 4-bit rollout and of the two ends of the policy, as
measurable cases.

Kinds (one pass each):

  layer      a linear layer in microscaled 4-bit floating point: X in bf16
             quantized per token, times weights laid out once, Y in bf16
  weights    a weight (or a batch of activations) as MXFP4: E2M1 codes with a
             power-of-two scale per 32 elements of a row (that of the largest
             magnitude over 4), and the bf16 values that they stand for
  embedding  rows of the embedding table for a batch of tokens, scaled
  embedding_backward
             the table's gradient over one or two micro-batches
  top        log-probabilities of the taken tokens, entropies, and the k most
             probable alternatives with their log-probabilities

Hidden and FFN sizes are those of perf/cases.py (4096 -> 12288, 5120 ->
17408), token counts go from a decode step to a 16K-token training step.
Scales come as bytes (the exponent + 127), in the layout [P / 256][rows][8]
for rows of P elements, P being the row's length filled up to a multiple of 256.
"""
import math

import torch

own = False

BF16 = torch.bfloat16
# The magnitudes of E2M1's codes 0 .. 7; bit 3 is the sign.
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # Rollout, a decode step of eight sequences: up projection of an 8B layer, weight bytes count.
        dict(name="layer_decode8", kind="layer", M=8, K=4096, N=12288),
        # Rollout, a decode step of 64 sequences: the 14B layer's way down.
        dict(name="layer_decode64", kind="layer", M=64, K=17408, N=5120),
        # Rollout prefill of a ragged number of tokens, 14B layer.
        dict(name="layer_prefill", kind="layer", M=3001, K=5120, N=17408),
        # Scoring of one 16K-token sequence.
        dict(name="layer_score", kind="layer", M=16384, K=4096, N=12288),
        # After an update: one projection's weights for the rollout.
        dict(name="weights_update", kind="weights", rows=12288, cols=4096),
        # A short ragged batch, rows that end inside a unit.
        dict(name="weights_ragged", kind="weights", rows=1001, cols=5000),
        # Rollout, a decode step of eight sequences: launch latency.
        dict(name="embedding_decode8", kind="embedding", T=8, V=131072, C=4096, dtype="bf16", scale=1.0),
        # Training, one 16K-token sequence, table in bf16, embeddings scaled by sqrt(C).
        dict(name="embedding_train", kind="embedding", T=16384, V=131072, C=5120, dtype="bf16", scale=71.5541752799933),
        # The table's whole gradient in 32 bits: its rows of zeros are most of the work.
        dict(name="embedding_backward_train", kind="embedding_backward", T=16384, V=131072, C=4096, dtype="f32",
             batches=1, scale=1.0),
        # A small vocabulary, bf16 gradient, two ragged micro-batches one after the other.
        dict(name="embedding_backward_accumulated", kind="embedding_backward", T=5003, V=32000, C=2048, dtype="bf16",
             batches=2, scale=45.254833995939045),
        # Rollout, one step of 64 sequences with twenty alternatives.
        dict(name="top_decode64", kind="top", T=64, V=131072, k=20, dtype="bf16", temperature=1.0),
        # A scored prompt of 2048 tokens with five alternatives, a vocabulary that is no multiple of anything, 32 bits.
        dict(name="top_prompt_f32", kind="top", T=2048, V=50021, k=5, dtype="f32", temperature=0.7),
    ]


def draw(rng):
    def log(lo, hi, step=1):
        return max(step, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)

    while True:
        kind = rng.choice(("layer", "layer", "layer", "weights", "embedding", "embedding_backward",
                           "embedding_backward", "top", "top"))
        if kind == "layer":
            case = dict(kind=kind, M=log(1, 16384), K=log(128, 17408, 32), N=log(256, 17408, 4))
        elif kind == "weights":
            case = dict(kind=kind, rows=log(1, 16384), cols=log(32, 17408, rng.choice((1, 32, 256))))
        elif kind == "embedding":
            C = log(256, 8192, 16)
            case = dict(kind=kind, T=log(1, 16384), V=log(8000, 160000), C=C, dtype=rng.choice(("bf16", "bf16", "f32")),
                        scale=rng.choice((1.0, math.sqrt(C))))
        elif kind == "embedding_backward":
            C = log(256, 8192, 16)
            case = dict(kind=kind, T=log(1, 40000), V=log(8000, 160000), C=C, dtype=rng.choice(("f32", "bf16")),
                        batches=rng.choice((1, 2)), scale=rng.choice((1.0, math.sqrt(C))))
        else:
            case = dict(kind=kind, T=log(1, 2048), V=log(8000, 160000), k=rng.choice((1, 2, 5, 8, 20, 64)),
                        dtype=rng.choice(("bf16", "bf16", "f32")), temperature=rng.choice((1.0, 1.0, 0.7)))
        most = [work(c) for c in listed() if c["kind"] == kind]
        cost = work(case)
        if all(cost[u] <= max(m[u] for m in most) for u in ("bytes", "flops")):
            return case


def _padded(cols):
    return -(-cols // 256) * 256


def work(case):
    """Inputs read once, outputs written once, and the operations on them (of
    the matrix products two per multiplication and addition).  Of a table only
    the rows that tokens name are read; distinct ones at most as many as tokens."""
    kind = case["kind"]
    if kind == "layer":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2.0 * M * K + N * K * 17.0 / 32 + 2.0 * M * N, "flops": 2.0 * M * N * K}
    if kind == "weights":
        n = case["rows"] * case["cols"]
        return {"bytes": 2.0 * n + n / 32.0 + 2.0 * n, "flops": 4.0 * n}
    if kind == "embedding":
        n = case["T"] * case["C"]
        return {"bytes": n * (2.0 + (2.0 if case["dtype"] == "bf16" else 4.0)) + 8.0 * case["T"], "flops": 1.0 * n}
    if kind == "embedding_backward":
        n = case["batches"] * case["T"] * case["C"]
        size = 4.0 if case["dtype"] == "f32" else 2.0
        return {"bytes": 2.0 * n + case["V"] * case["C"] * size + 8.0 * case["batches"] * case["T"], "flops": 1.0 * n}
    n = case["T"] * case["V"]
    return {"bytes": n * (2.0 if case["dtype"] == "bf16" else 4.0) + case["T"] * (16.0 + 12.0 * case["k"]),
            "flops": 7.0 * n}


def _exponents(v):
    """Exponents of the units' scales: that of the largest magnitude less that of the largest
    code, 6 = 1.5 * 2^2, at least -127, 0 for a unit of zeros; v fp32 [rows, P], [rows, P / 32]."""
    m, e = torch.frexp(v.view(v.shape[0], -1, 32).abs().amax(dim=2))  # (amax = m 2^e, m in [0.5, 1))
    return torch.where(m == 0, torch.zeros_like(e), torch.clamp(e - 3, min=-127))


def _filled(x):
    """x in fp32, its rows filled up with zeros to whole pieces of 256."""
    return torch.nn.functional.pad(x.float(), (0, _padded(x.shape[1]) - x.shape[1]))


def _power(k):
    """2^k in fp32, exactly, for whole k from -126 to 127."""
    return ((k + 127).to(torch.int32) << 23).view(torch.float32)


def _rounded(v):
    """fp32 values to the nearest of E2M1, ties to the even code, magnitudes above 6 to 6."""
    a = v.abs().clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step, v)


def _quantized(x):
    """(E2M1 values [rows, P] in fp32, exponents [rows, P / 32]) of x."""
    v = _filled(x)
    k = _exponents(v)
    return _rounded(v * _power(-k).repeat_interleave(32, dim=1)), k


def _scale_bytes(k):
    """Exponents [rows, P / 32] as bytes in the library's layout [P / 256][rows][8]."""
    return (k + 127).to(torch.uint8).view(k.shape[0], -1, 8).permute(1, 0, 2).reshape(-1)


def _packed(values):
    """The codes of E2M1 values, two a byte, the first in the low half."""
    a = values.abs()
    code = torch.where(a < 2.0, a * 2.0, torch.where(a < 4.0, a + 2.0, a * 0.5 + 4.0)).to(torch.uint8)
    code += torch.signbit(values).to(torch.uint8) * 8
    return code[:, 0::2] + code[:, 1::2] * 16


def _values(codes, scales):
    """What codes [rows, P / 2] with scale bytes in the library's layout stand for, in fp32."""
    rows = codes.shape[0]
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), dim=2).view(rows, -1)
    k = scales.view(-1, rows, 8).permute(1, 0, 2).reshape(rows, -1).to(torch.int32) - 127
    return v * _power(k).repeat_interleave(32, dim=1)


def prepare(case, seed):
    """Hidden states N(0, 1) with 1% of the channels fifty times as large,
    projection weights N(0, 0.02); tokens with frequencies of 1 / rank, one in
    fifty (of a training batch) padding: -1; table N(0, 0.02), output gradients
    N(0, 1e-3); logits N(0, 2) with tokens drawn from their softmax."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(sigma)

    def stream(rows, cols):
        x = normal(rows, cols)
        x[:, torch.randperm(cols, generator=g, device="cuda")[: max(1, round(0.01 * cols))]] *= 50.0
        return x.to(BF16)

    kind = case["kind"]
    s = dict(case=case)
    if kind == "layer":
        s["x"] = stream(case["M"], case["K"])
        values, k = _quantized(normal(case["N"], case["K"], sigma=0.02).to(BF16))
        s["w"], s["sw"] = _packed(values), _scale_bytes(k)
    elif kind == "weights":
        s["x"] = normal(case["rows"], case["cols"], sigma=0.02).to(BF16)
    elif kind in ("embedding", "embedding_backward"):
        T, V, C, n = case["T"], case["V"], case["C"], case.get("batches", 1)
        tokens = torch.exp(torch.rand((n, T), generator=g, device="cuda").double() * math.log(V)).long() - 1
        if T >= 16:
            tokens[torch.rand((n, T), generator=g, device="cuda") < 0.02] = -1
        s["tokens"] = [t.contiguous() for t in tokens]
        if kind == "embedding":
            w = normal(V, C, sigma=0.02)
            s["weight"] = w.to(BF16) if case["dtype"] == "bf16" else w
        else:
            s["dy"] = [normal(T, C, sigma=1e-3).to(BF16) for _ in range(n)]
    else:
        T, V, t = case["T"], case["V"], case["temperature"]
        x = normal(T, V, sigma=2.0).to(BF16 if case["dtype"] == "bf16" else torch.float32)
        s["tokens"] = torch.empty(T, dtype=torch.int64, device="cuda")
        for r in range(0, T, 512):
            u = torch.rand((min(512, T - r), V), generator=g, device="cuda").clamp_(min=1e-20)
            s["tokens"][r:r + 512] = torch.argmax(x[r:r + 512].float() / t - torch.log(-torch.log(u)), dim=1)
        s["x"] = x
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2609_22870_amd as fp8q

    case = s["case"]
    kind = case["kind"]
    if kind == "layer":
        codes, scales = fp8q.quantize_mx4(s["x"])
        return dict(y=fp8q.gemm_mx4(codes, scales, s["w"], s["sw"]))
    if kind == "weights":
        codes, scales = fp8q.quantize_mx4(s["x"])
        return dict(values=fp8q.dequantize_mx4(codes, scales, case["cols"]), scales=scales)
    if kind == "embedding":
        return dict(y=fp8q.embedding(s["weight"], s["tokens"][0], case["scale"]))
    if kind == "embedding_backward":
        dtype = torch.float32 if case["dtype"] == "f32" else BF16
        dw = fp8q.embedding_backward(s["dy"][0], s["tokens"][0], case["V"], case["scale"], dtype=dtype)
        for dy, tokens in zip(s["dy"][1:], s["tokens"][1:]):
            fp8q.embedding_backward(dy, tokens, case["V"], case["scale"], dtype=dtype, dweight=dw, accumulate=True)
        return dict(dw=dw)
    logp, entropy, ids, top = fp8q.top_logprobs(s["x"], s["tokens"], case["k"], temperature=case["temperature"])
    return dict(logp=logp, entropy=entropy, ids=ids, top=top)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "layer":
        q, k = _quantized(s["x"])
        x = q * _power(k).repeat_interleave(32, dim=1)
        return dict(y=(x @ _values(s["w"], s["sw"]).t()).to(BF16))
    if kind == "weights":
        q, k = _quantized(s["x"])
        v = q * _power(k).repeat_interleave(32, dim=1)
        return dict(values=v[:, : case["cols"]].to(BF16), scales=_scale_bytes(k))
    if kind == "embedding":
        t = s["tokens"][0]
        y = s["weight"][t.clamp(min=0)].float() * case["scale"]
        return dict(y=torch.where((t >= 0)[:, None], y, torch.zeros_like(y)).to(BF16))
    if kind == "embedding_backward":
        dtype = torch.float32 if case["dtype"] == "f32" else BF16
        dw = None
        for dy, t in zip(s["dy"], s["tokens"]):
            d = torch.zeros((case["V"], case["C"]), device="cuda")
            d.index_add_(0, t.clamp(min=0), dy.float() * (t >= 0)[:, None])
            d *= case["scale"]
            dw = (d if dw is None else dw.float() + d).to(dtype)
        return dict(dw=dw)
    x = s["x"].float()
    # keys of the logits' order, then of the lowest index; all different
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    V = case["V"]
    keys = bits.to(torch.int64) * 2 ** 32 + torch.arange(V - 1, -1, -1, device=x.device)
    ids = V - 1 - (torch.topk(keys, case["k"], dim=1).values & 0xFFFFFFFF)
    del bits, keys
    z = x / case["temperature"]
    most = z.amax(dim=1, keepdim=True)
    p = torch.exp(z - most)
    total = p.sum(dim=1, keepdim=True)
    lse = most + torch.log(total)
    p /= total
    return dict(logp=(torch.gather(z, 1, s["tokens"][:, None]) - lse)[:, 0], entropy=lse[:, 0] - (p * z).sum(dim=1),
                ids=ids, top=torch.gather(z, 1, ids) - lse)


def exact(case, seed):
    """run()'s results in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    f64 = torch.float64

    def nearest(x):
        """x in MXFP4, as the values that its codes stand for: in each unit of 32 the nearest of
        the levels times 2^(floor(log2 amax) - 2)."""
        rows, cols = x.shape
        u = torch.nn.functional.pad(x.to(f64), (0, -cols % 32)).view(rows, -1, 32)
        amax = u.abs().amax(dim=2, keepdim=True)
        # (the exponent field of a 64-bit number; its power of two from the field again)
        k = torch.where(amax == 0, 0, ((amax.view(torch.int64) >> 52) - 1025).clamp(min=-127))
        scale = ((k + 1023) << 52).view(f64)
        level = torch.tensor(LEVELS, dtype=f64, device="cuda")
        middle = (level[1:] + level[:-1]) / 2.0
        a = (u / scale).abs()
        low = torch.bucketize(a, middle)  # (a middle goes down here)
        up = (low < 7) & (a == middle[low.clamp(max=6)]) & (low % 2 == 1)
        return (torch.sign(u) * level[low + up.long()] * scale).view(rows, -1)[:, :cols]

    if kind == "layer":
        M, K, N = case["M"], case["K"], case["N"]
        level = torch.tensor(LEVELS, dtype=f64, device="cuda")
        level = torch.cat((level, -level))
        w = torch.stack((level[(s["w"] % 16).long()], level[(s["w"] // 16).long()]), dim=-1).view(N, -1, 32)
        sw = ((s["sw"].view(-1, N, 8).long() - 127 + 1023) << 52).view(f64).transpose(0, 1).reshape(N, -1, 1)
        w = (w * sw).view(N, -1)[:, :K].t().contiguous()
        x = nearest(s["x"])
        return dict(y=torch.cat([torch.mm(x[r:r + 4096], w) for r in range(0, M, 4096)]))
    if kind == "weights":
        return dict(values=nearest(s["x"]), scales=None)
    if kind == "embedding":
        t = s["tokens"][0]
        y = torch.zeros((case["T"], case["C"]), dtype=f64, device="cuda")
        y[t >= 0] = s["weight"][t[t >= 0]].to(f64) * case["scale"]
        return dict(y=y)
    if kind == "embedding_backward":
        dw = torch.zeros((case["V"], case["C"]), dtype=f64, device="cuda")
        for dy, t in zip(s["dy"], s["tokens"]):
            dw.index_add_(0, t[t >= 0], dy[t >= 0].to(f64), alpha=case["scale"])
        return dict(dw=dw)
    T = case["T"]
    logp, entropy = torch.empty(T, dtype=f64, device="cuda"), torch.empty(T, dtype=f64, device="cuda")
    top = torch.empty((T, case["k"]), dtype=f64, device="cuda")
    for r in range(0, T, 256):
        rows = slice(r, min(T, r + 256))
        lp = torch.log_softmax(s["x"][rows].to(f64) / case["temperature"], dim=1)
        logp[rows] = torch.gather(lp, 1, s["tokens"][rows, None])[:, 0]
        entropy[rows] = -(lp.exp() * lp).sum(dim=1)
        top[rows] = torch.sort(lp, dim=1, descending=True).values[:, : case["k"]]
    return dict(logp=logp, entropy=entropy, ids=None, top=top)
