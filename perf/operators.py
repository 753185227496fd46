"""The operators around the FP8 linear layers of a policy's training step and
rollout, as measurable cases.

Kinds (one pass each):

  norm           h = x + residual, RMS norm of h, FP8 output with scales (per
                 1x128 block or per row) or bf16 output
  norm_backward  its gradients: of x (and of the residual: the same) and of
                 the norm's weight
  gated          H = silu(X Wg^T) * (X Wu^T) from FP8 operands; out "bf16":
                 H itself; "down": H in FP8 and the down projection of it;
                 pre: the pre-activations are kept for the backward pass
  gated_backward the gradients of both pre-activations in the two FP8 layouts
                 that the data- and weight-gradient GEMMs take
  requantize     an activation kept in FP8 (1x128 units) as the weight
                 gradient's operand: transposed, in 128x1 units
  logprobs       log-probabilities of the taken tokens, and entropies
  loss           clipped policy loss with a KL term: loss, log-probabilities,
                 entropies and the gradient in the logits

Hidden and FFN sizes are those of perf/cases.py (4096 -> 12288, 5120 ->
17408), token counts go from a decode step to a 16K-token training step.
Codes are returned as the FP8 values they stand for.
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
EPS = 1e-6
# The clipping bounds (ratio), the KL coefficient of the loss cases.
CLIP_LOW, CLIP_HIGH, BETA = 0.8, 1.24, 0.05


def listed():
    return [
        # Rollout, a decode step of eight sequences: the norm in front of a projection, launch latency.
        dict(name="norm_decode8", kind="norm", rows=8, cols=4096, residual=True, out="block"),
        # Training, one 16K-token sequence: residual stream in, FP8 operand and residual stream out.
        dict(name="norm_train", kind="norm", rows=16384, cols=5120, residual=True, out="block"),
        # The same layer's backward pass.
        dict(name="norm_backward_train", kind="norm_backward", rows=16384, cols=4096, residual=True),
        # Rollout, a decode step of eight sequences: gate and up projections of an 8B layer.
        dict(name="gated_decode8", kind="gated", M=8, K=4096, F=12288, out="bf16", pre=False),
        # Rollout prefill of a ragged number of tokens, 14B layer, the whole block.
        dict(name="gated_prefill", kind="gated", M=3001, K=5120, F=17408, out="down", pre=False),
        # Training forward of the whole block, pre-activations kept.
        dict(name="gated_train", kind="gated", M=16384, K=4096, F=12288, out="down", pre=True),
        # Its activation's backward pass.
        dict(name="gated_backward_train", kind="gated_backward", M=16384, F=12288, e5m2=False),
        # The kept input of a weight gradient: a whole sequence of FFN activations ...
        dict(name="requantize_train", kind="requantize", rows=16384, cols=12288),
        # ... and a short ragged batch of hidden states.
        dict(name="requantize_ragged", kind="requantize", rows=1001, cols=5120),
        # Rollout: log-probabilities of one step of 64 sequences.
        dict(name="logprobs_decode64", kind="logprobs", T=64, V=131072, dtype="bf16", temperature=1.0),
        # Training: the loss of a micro-batch of 8192 tokens over a large vocabulary.
        dict(name="loss_train", kind="loss", T=8192, V=131072, dtype="bf16", temperature=1.0),
        # A short micro-batch in 32 bits, a vocabulary that is no multiple of anything.
        dict(name="loss_small_f32", kind="loss", T=33, V=50021, dtype="f32", temperature=0.7),
    ]


def draw(rng):
    def log(lo, hi, step=1):
        return max(step, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)

    while True:
        kind = rng.choice(("norm", "norm", "norm_backward", "gated", "gated", "gated", "gated_backward", "requantize",
                           "logprobs", "loss", "loss"))
        if kind == "norm":
            out = rng.choice(("block", "block", "row", "bf16"))
            case = dict(kind=kind, rows=log(1, 16384), cols=log(256, 8192, 128 if out == "block" else 16),
                        residual=rng.random() < 0.7, out=out)
        elif kind == "norm_backward":
            case = dict(kind=kind, rows=log(16, 16384), cols=log(256, 8192, 16), residual=rng.random() < 0.7)
        elif kind == "gated":
            out = rng.choice(("bf16", "down"))
            case = dict(kind=kind, M=log(1, 16384), K=log(256, 8192, 128), F=log(512, 16384, 128), out=out,
                        pre=rng.random() < 0.5)
        elif kind == "gated_backward":
            case = dict(kind=kind, M=log(64, 16384), F=log(512, 16384, 128), e5m2=rng.random() < 0.4)
        elif kind == "requantize":
            case = dict(kind=kind, rows=log(64, 16384), cols=log(256, 16384, 128))
        else:
            lo, hi = (1, 512) if kind == "logprobs" else (8, 8192)
            case = dict(kind=kind, T=log(lo, hi), V=log(8000, 160000), dtype=rng.choice(("bf16", "bf16", "f32")),
                        temperature=rng.choice((1.0, 1.0, 0.7)))
        name = {"norm": "norm_train", "norm_backward": "norm_backward_train", "gated": "gated_train",
                "gated_backward": "gated_backward_train", "requantize": "requantize_train"}.get(kind, "loss_train")
        most = work(next(c for c in listed() if c["name"] == name))
        cost = work(case)
        # (3072 is no width of the layers that the package is used for)
        if 3072 not in case.values() and cost["bytes"] <= most["bytes"] and cost["flops"] <= most["flops"]:
            return case


def work(case):
    """Inputs read once, outputs written once, and the operations on them (of
    the matrix products two per multiplication and addition)."""
    kind = case["kind"]
    if kind == "norm":
        n, r = case["rows"] * case["cols"], case["residual"]
        out = {"block": 1.0 + 4.0 / 128, "row": 1.0, "bf16": 2.0}[case["out"]]
        return {"bytes": n * (2.0 + (4.0 if r else 0.0) + out) + 8.0 * case["rows"] + 2.0 * case["cols"],
                "flops": 8.0 * n}
    if kind == "norm_backward":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (6.0 + (2.0 if case["residual"] else 0.0)) + 4.0 * case["rows"] + 6.0 * case["cols"],
                "flops": 10.0 * n}
    if kind == "gated":
        M, K, F = case["M"], case["K"], case["F"]
        b, f = M * K + 2.0 * F * K + 4.0 * M * K / 128, 4.0 * M * K * F
        b += 4.0 * M * F if case["pre"] else 0.0
        if case["out"] == "down":
            return {"bytes": b + M * F + F * K + 2.0 * M * K, "flops": f + 2.0 * M * K * F}
        return {"bytes": b + 2.0 * M * F, "flops": f}
    if kind == "gated_backward":
        n = case["M"] * case["F"]
        return {"bytes": n * (10.0 + 16.0 / 128), "flops": 20.0 * n}
    if kind == "requantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2.0 + 8.0 / 128), "flops": 4.0 * n}
    n = case["T"] * case["V"]
    size = 2.0 if case["dtype"] == "bf16" else 4.0
    return {"bytes": n * size * (2.0 if kind == "loss" else 1.0) + 40.0 * case["T"],
            "flops": n * (9.0 if kind == "loss" else 6.0)}


def _units(v):
    """Scales of v's 1x128 units: fp32(amax / 448), 1 for a zero unit; [rows, cols / 128]."""
    s = v.view(v.shape[0], -1, 128).abs().amax(dim=2) / 448.0
    return torch.where(s == 0, torch.ones_like(s), s)


def _codes(v, s, e5m2=False):
    """The FP8 values nearest to v / s."""
    top = 57344.0 if e5m2 else 448.0
    return torch.clamp(v / s, -top, top).to(torch.float8_e5m2 if e5m2 else F8)


def _block_codes(v):
    """v as FP8 values in 1x128 units and its scales in the library's layout [cols / 128][rows]."""
    s = _units(v)
    return _codes(v, s.repeat_interleave(128, dim=1)), s.t().reshape(-1)


def _column_codes(v, e5m2=False):
    """v's transpose as FP8 values in units of 128 rows (the last one filled up with zeros), and
    the scales [rows / 128][cols]."""
    v = torch.nn.functional.pad(v, (0, 0, 0, -v.shape[0] % 128))
    s = v.view(-1, 128, v.shape[1]).abs().amax(dim=1) / (57344.0 if e5m2 else 448.0)
    s = torch.where(s == 0, torch.ones_like(s), s)
    return _codes(v, s.repeat_interleave(128, dim=0), e5m2).t().contiguous(), s.reshape(-1)


def _values(codes, scales):
    """What FP8 codes with 1x128 scales stand for."""
    s = scales.view(-1, codes.shape[0]).t().repeat_interleave(128, dim=1)
    return codes.view(F8).float() * s


def _weight_values(codes, scales):
    """The same with 128x128 scales."""
    n, k = codes.shape
    return codes.view(F8).float() * scales.view(n // 128, k // 128).repeat_interleave(128, 0).repeat_interleave(128, 1)


def _weight(rows, cols, g):
    """An FP8 weight laid out once: codes and 128x128 scales of N(0, 0.02)."""
    w = torch.randn((rows, cols), generator=g, device="cuda").mul_(0.02)
    s = w.view(rows // 128, 128, cols // 128, 128).abs().amax(dim=(1, 3)) / 448.0
    q = _codes(w, s.repeat_interleave(128, 0).repeat_interleave(128, 1))
    return q.view(torch.uint8), s.reshape(-1)


def prepare(case, seed):
    """Residual streams N(0, 1) with 1% of the channels fifty times as large,
    norm weights around 1, projection weights N(0, 0.02), output gradients
    N(0, 1e-3); logits N(0, 2) with tokens drawn from their softmax, one token
    in seven outside the response (weight 0)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    bf16 = torch.bfloat16

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(sigma)

    def stream(rows, cols):
        x = normal(rows, cols)
        x[:, torch.randperm(cols, generator=g, device="cuda")[: max(1, round(0.01 * cols))]] *= 50.0
        return x.to(bf16)

    kind = case["kind"]
    s = dict(case=case)
    if kind in ("norm", "norm_backward"):
        rows, cols = case["rows"], case["cols"]
        s.update(x=stream(rows, cols), w=(1.0 + 0.1 * normal(cols)).to(bf16))
        if kind == "norm":
            s["residual"] = normal(rows, cols).to(bf16) if case["residual"] else None
        else:
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(dim=1) + EPS)
            s["dy"] = normal(rows, cols, sigma=1e-3).to(bf16)
            s["dres"] = normal(rows, cols, sigma=1e-3).to(bf16) if case["residual"] else None
    elif kind == "gated":
        M, K, F = case["M"], case["K"], case["F"]
        q, s["sx"] = _block_codes(stream(M, K).float())
        s["x"] = q.view(torch.uint8)
        s["w"], s["sw"] = _weight(2 * F, K, g)
        if case["out"] == "down":
            s["wd"], s["swd"] = _weight(K, F, g)
    elif kind == "gated_backward":
        s["pre"] = normal(case["M"], 2 * case["F"], sigma=2.0).to(bf16)
        s["dh"] = normal(case["M"], case["F"], sigma=1e-3).to(bf16)
    elif kind == "requantize":
        q, s["sx"] = _block_codes(stream(case["rows"], case["cols"]).float())
        s["x"] = q.view(torch.uint8)
    else:
        T, V, t = case["T"], case["V"], case["temperature"]
        x = torch.empty((T, V), dtype=bf16 if case["dtype"] == "bf16" else torch.float32, device="cuda")
        tokens = torch.empty(T, dtype=torch.int64, device="cuda")
        logp = torch.empty(T, device="cuda")
        for r in range(0, T, 1024):
            x[r:r + 1024] = normal(min(1024, T - r), V, sigma=2.0)
            z = x[r:r + 1024].float() / t
            u = torch.rand(z.shape, generator=g, device="cuda").clamp_(min=1e-20)
            tokens[r:r + 1024] = torch.argmax(z - torch.log(-torch.log(u)), dim=1)
            logp[r:r + 1024] = torch.gather(z, 1, tokens[r:r + 1024, None])[:, 0] - torch.logsumexp(z, dim=1)
        s.update(x=x, tokens=tokens)
        if kind == "loss":
            # ratios exp(N(0, 0.15)); none within 1e-3 of a bound, where the derivative jumps and
            # a rounding decides which side's is the answer
            d = normal(T, sigma=0.15)
            for b in (math.log(CLIP_LOW), math.log(CLIP_HIGH)):
                d = torch.where((d - b).abs() < 1e-3, torch.full_like(d, b + 2e-3), d)
            live = torch.rand(T, generator=g, device="cuda") >= 1.0 / 7.0
            live[0] = True
            s.update(old=logp - d, ref=logp + normal(T, sigma=0.2), adv=0.3 + normal(T),
                     w_tis=torch.exp(normal(T, sigma=0.1)).clamp_(max=2.0), weight=live.float() / live.sum())
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2609_22870_amd as fp8q

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        if case["out"] == "bf16":
            y, h, rstd = fp8q.rmsnorm(s["x"], s["w"], EPS, residual=s["residual"])
            return dict(y=y, h=h, rstd=rstd)
        g = fp8q.ROW if case["out"] == "row" else fp8q.BLOCK_1x128
        codes, scales, h, rstd = fp8q.rmsnorm_quantize(s["x"], s["w"], EPS, g, residual=s["residual"])
        return dict(codes=codes.view(F8), scales=scales, h=h, rstd=rstd)
    if kind == "norm_backward":
        dx, dw = fp8q.rmsnorm_backward(s["dy"], s["x"], s["rstd"], s["w"], dres=s["dres"])
        return dict(dx=dx, dw=dw)
    if kind == "gated":
        if case["out"] == "bf16":
            h, pre = fp8q.gemm_gated(s["x"], s["sx"], s["w"], s["sw"], save=case["pre"])
            return dict(h=h, pre=pre)
        codes, scales, pre = fp8q.gemm_gated_quantized(s["x"], s["sx"], s["w"], s["sw"], save=case["pre"])
        y = fp8q.gemm(codes, scales, fp8q.BLOCK_1x128, s["wd"], s["swd"], fp8q.BLOCK_128x128)
        return dict(h=codes.view(F8), pre=pre, y=y)
    if kind == "gated_backward":
        cr, sr, ct, st = fp8q.gated_backward(s["dh"], s["pre"], e5m2=case["e5m2"])
        f8 = torch.float8_e5m2 if case["e5m2"] else F8
        return dict(codes=cr.view(f8), scales=sr, codes_t=ct.view(f8), scales_t=st)
    if kind == "requantize":
        codes, scales = fp8q.requantize_transposed(s["x"], s["sx"])
        return dict(codes=codes.view(F8), scales=scales)
    if kind == "logprobs":
        logp, entropy = fp8q.token_logprobs(s["x"], s["tokens"], temperature=case["temperature"])
        return dict(logp=logp, entropy=entropy)
    loss, dlogits, logp, entropy = fp8q.policy_loss(s["x"], s["tokens"], s["old"], s["adv"], s["weight"], CLIP_LOW,
                                                    CLIP_HIGH, beta=BETA, logp_ref=s["ref"], w_tis=s["w_tis"],
                                                    temperature=case["temperature"])
    return dict(loss=loss, dlogits=dlogits, logp=logp, entropy=entropy)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        # the norm is that of the residual stream as it is kept, in bf16
        h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(torch.bfloat16)
        v = h.float()
        rstd = 1.0 / torch.sqrt((v * v).mean(dim=1) + EPS)
        y = v * rstd[:, None] * s["w"].float()
        if case["out"] == "bf16":
            return dict(y=y.to(torch.bfloat16), h=h, rstd=rstd)
        if case["out"] == "row":
            scales = y.abs().amax(dim=1) / 448.0
            codes = _codes(y, scales[:, None])
        else:
            codes, scales = _block_codes(y)
        return dict(codes=codes, scales=scales, h=h, rstd=rstd)
    if kind == "norm_backward":
        dy, xhat = s["dy"].float(), s["x"].float() * s["rstd"][:, None]
        u = dy * s["w"].float()
        dx = s["rstd"][:, None] * (u - xhat * (u * xhat).mean(dim=1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return dict(dx=dx.to(torch.bfloat16), dw=(dy * xhat).sum(dim=0))
    if kind == "gated":
        z = _values(s["x"], s["sx"]) @ _weight_values(s["w"], s["sw"]).t()
        gate, up = z[:, : case["F"]], z[:, case["F"]:]
        h = (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)
        pre = z.to(torch.bfloat16) if case["pre"] else None
        if case["out"] == "bf16":
            return dict(h=h, pre=pre)
        codes, scales = _block_codes(h.float())
        y = _values(codes, scales) @ _weight_values(s["wd"], s["swd"]).t()
        return dict(h=codes, pre=pre, y=y.to(torch.bfloat16))
    if kind == "gated_backward":
        F = case["F"]
        gate, up, dh = s["pre"][:, :F].float(), s["pre"][:, F:].float(), s["dh"].float()
        sig = 1.0 / (1.0 + torch.exp(-gate))
        d = torch.cat((dh * up * sig * (1.0 + gate * (1.0 - sig)), dh * gate * sig), dim=1)
        top = 57344.0 if case["e5m2"] else 448.0
        scales = d.view(d.shape[0], -1, 128).abs().amax(dim=2) / top
        scales = torch.where(scales == 0, torch.ones_like(scales), scales)
        codes = _codes(d, scales.repeat_interleave(128, dim=1), case["e5m2"])
        codes_t, scales_t = _column_codes(d, case["e5m2"])
        return dict(codes=codes, scales=scales.t().reshape(-1), codes_t=codes_t, scales_t=scales_t)
    if kind == "requantize":
        codes, scales = _column_codes(_values(s["x"], s["sx"]))
        return dict(codes=codes, scales=scales)
    z = s["x"].float() / case["temperature"]
    top = z.amax(dim=1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    p /= total
    logp = torch.gather(z, 1, s["tokens"][:, None])[:, 0] - lse
    entropy = lse - (p * z).sum(dim=1)
    if kind == "logprobs":
        return dict(logp=logp, entropy=entropy)
    del z
    live = s["weight"] != 0
    r, d = torch.exp(logp - s["old"]), s["ref"] - logp
    a, b = r * s["adv"], torch.clamp(r, CLIP_LOW, CLIP_HIGH) * s["adv"]
    term = -s["w_tis"] * torch.minimum(a, b) + BETA * (torch.exp(d) - d - 1.0)
    slope = torch.where(a <= b, -s["w_tis"] * a, torch.zeros_like(a)) + BETA * (1.0 - torch.exp(d))
    k = torch.where(live, s["weight"] * slope, torch.zeros_like(slope)) / case["temperature"]
    p *= -k[:, None]
    p.scatter_add_(1, s["tokens"][:, None], k[:, None])
    zero = torch.zeros_like(logp)
    return dict(loss=torch.where(live, s["weight"] * term, zero).sum().reshape(1), dlogits=p.to(s["x"].dtype),
                logp=torch.where(live, logp, zero), entropy=torch.where(live, entropy, zero))


def exact(case, seed):
    """run()'s results in 64 bits (for FP8 codes the values before their rounding)."""
    s = prepare(case, seed)
    kind = case["kind"]
    f64 = torch.float64

    def blocks(v, top):
        """(values of 1x128 units over their scales, scales [cols / 128][rows])"""
        u = v.reshape(v.shape[0], -1, 128)
        k = u.abs().amax(dim=2) / top
        k = torch.where(k == 0, torch.ones_like(k), k)
        return (u / k[:, :, None]).reshape(v.shape), k.t().contiguous().reshape(-1)

    def columns(v, top):
        q, k = blocks(torch.nn.functional.pad(v, (0, 0, 0, -v.shape[0] % 128)).t().contiguous(), top)
        return q, k

    def layer(codes, scales, weight, wscales):
        """The product of the values that both operands' codes stand for."""
        a = codes.view(F8).to(f64) * scales.to(f64).view(-1, codes.shape[0]).t().repeat_interleave(128, 1)
        n, k = weight.shape
        b = weight.view(F8).to(f64).view(n // 128, 128, k // 128, 128)
        b = (b * wscales.to(f64).view(n // 128, 1, k // 128, 1)).view(n, k)
        return torch.cat([torch.mm(a[r:r + 4096], b.t()) for r in range(0, a.shape[0], 4096)])

    if kind == "norm":
        h = s["x"]
        if s["residual"] is not None:
            h = (h.to(f64) + s["residual"].to(f64)).to(torch.bfloat16)
        v = h.to(f64)
        rms = torch.sqrt(v.pow(2).sum(dim=1) / v.shape[1] + EPS)
        y = v / rms[:, None] * s["w"].to(f64)
        if case["out"] == "bf16":
            return dict(y=y, h=h.to(f64), rstd=1.0 / rms)
        if case["out"] == "row":
            top = y.abs().amax(dim=1) / 448.0
            return dict(codes=y / top[:, None], scales=top, h=h.to(f64), rstd=1.0 / rms)
        codes, scales = blocks(y, 448.0)
        return dict(codes=codes, scales=scales, h=h.to(f64), rstd=1.0 / rms)
    if kind == "norm_backward":
        # from the derivative of h_i / rms w_i: the sum over i of dy_i w_i (delta_ij rstd - h_i h_j rstd^3 / n)
        h, dy, w, rstd = s["x"].to(f64), s["dy"].to(f64), s["w"].to(f64), s["rstd"].to(f64)[:, None]
        dot = (dy * w * h).sum(dim=1, keepdim=True)
        dx = dy * w * rstd - h * rstd.pow(3) * dot / h.shape[1]
        if s["dres"] is not None:
            dx += s["dres"].to(f64)
        return dict(dx=dx, dw=(dy * h * rstd).sum(dim=0))
    if kind == "gated":
        z = layer(s["x"], s["sx"], s["w"], s["sw"])
        h = z[:, : case["F"]] * torch.sigmoid(z[:, : case["F"]]) * z[:, case["F"]:]
        pre = z if case["pre"] else None
        if case["out"] == "bf16":
            return dict(h=h, pre=pre)
        codes, scales = blocks(h, 448.0)
        n, k = s["wd"].shape
        wd = s["wd"].view(F8).to(f64).view(n // 128, 128, k // 128, 128)
        wd = (wd * s["swd"].to(f64).view(n // 128, 1, k // 128, 1)).view(n, k)
        return dict(h=codes, pre=pre, y=torch.cat([torch.mm(h[r:r + 4096], wd.t()) for r in range(0, h.shape[0], 4096)]))
    if kind == "gated_backward":
        F, top = case["F"], 57344.0 if case["e5m2"] else 448.0
        gate, up, dh = s["pre"][:, :F].to(f64), s["pre"][:, F:].to(f64), s["dh"].to(f64)
        sig = torch.sigmoid(gate)
        d = torch.cat((dh * up * (sig + gate * sig * (1.0 - sig)), dh * gate * sig), dim=1)
        codes, scales = blocks(d, top)
        codes_t, scales_t = columns(d, top)
        # (the columns' scales of a unit lie beside each other: [rows / 128][cols])
        return dict(codes=codes, scales=scales, codes_t=codes_t, scales_t=scales_t)
    if kind == "requantize":
        v = s["x"].view(F8).to(f64) * s["sx"].to(f64).view(-1, case["rows"]).t().repeat_interleave(128, 1)
        codes, scales = columns(v, 448.0)
        return dict(codes=codes, scales=scales)
    T, t = case["T"], case["temperature"]
    logp, entropy = torch.zeros(T, dtype=f64, device="cuda"), torch.zeros(T, dtype=f64, device="cuda")
    live = s["weight"] != 0 if kind == "loss" else torch.ones(T, dtype=torch.bool, device="cuda")
    dlogits = torch.zeros(s["x"].shape, dtype=f64, device="cuda") if kind == "loss" else None
    loss = 0.0
    for r in range(0, T, 1024):
        rows = slice(r, min(T, r + 1024))
        lp = torch.log_softmax(s["x"][rows].to(f64) / t, dim=1)
        on, tok = live[rows], s["tokens"][rows, None]
        mine = torch.gather(lp, 1, tok)[:, 0]
        logp[rows] = torch.where(on, mine, torch.zeros_like(mine))
        p = lp.exp()
        entropy[rows] = torch.where(on, -(p * lp).sum(dim=1), torch.zeros_like(mine))
        if kind == "loss":
            # per token and side: the derivative of -w min(rA, clip(r)A) is that of the smaller side
            a, w = s["adv"][rows].to(f64), s["w_tis"][rows].to(f64)
            ratio, off = torch.exp(mine - s["old"][rows].to(f64)), s["ref"][rows].to(f64) - mine
            bound = torch.where(a > 0, torch.full_like(a, CLIP_HIGH), torch.full_like(a, CLIP_LOW))
            cut = torch.where(a > 0, ratio > bound, ratio < bound)
            gain = torch.where(cut, bound, ratio) * a
            c = torch.where(on, s["weight"][rows].to(f64), torch.zeros_like(a))
            loss += float((c * (-w * gain + BETA * (torch.expm1(off) - off))).sum())
            k = c * (torch.where(cut, torch.zeros_like(a), -w * ratio * a) - BETA * torch.expm1(off)) / t
            dlogits[rows] = -k[:, None] * p
            dlogits[rows].scatter_add_(1, tok, k[:, None])
    if kind == "logprobs":
        return dict(logp=logp, entropy=entropy)
    return dict(loss=torch.tensor([loss], dtype=f64), dlogits=dlogits, logp=logp, entropy=entropy)
