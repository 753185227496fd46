"""Log-probabilities of the taken tokens and the clipped policy loss with its KL
term and gradient, from logits, against 64-bit references.

Tolerances.  A row's sum of exponentials is added in fp32 from positive terms, in
a thread at most 160 of them one after another and 16 levels across the row; each
exponential is good to 2^-22 plus 2^-24 of its exponent's magnitude R (the row's
range in base 2).  So log-probabilities are within e = (180 + 2 R) 2^-24 + 8 x
2^-24 (|logp| + |max z|), entropies within 4 R e, ratios and derivatives within a
few e of themselves."""
import math

import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, bf16_half, same, within

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LOW, HIGH, BETA = 0.8, 1.24, 0.05
# every kernel: a row in 256, 512 or 1024 threads, rows of more than the registers hold, rows over several workgroups
SHAPES = [(1, 1), (2, 3), (3, 8), (5, 100), (130, 1001), (200, 8191), (130, 9000), (150, 20001), (140, 40003),
          (129, 131072), (128, 180001), (1, 50021), (7, 70001), (3, 131072), (2, 300007)]


def batch(T, V, dtype, seed, t=1.0, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    x = (sigma * torch.randn(T, V, generator=g)).to(dtype)
    tokens = torch.randint(0, V, (T,), generator=g)
    lp = torch.log_softmax(x.to(F64) / t, dim=1).gather(1, tokens[:, None])[:, 0]
    d = 0.3 * torch.randn(T, generator=g, dtype=F64)
    for b in (math.log(LOW), math.log(HIGH)):  # (at a bound the derivative jumps)
        d = torch.where((d - b).abs() < 1e-3, torch.full_like(d, b + 2e-3), d)
    b = dict(logits=x, tokens=tokens, logp_old=(lp - d).float(), adv=torch.randn(T, generator=g),
             weight=torch.rand(T, generator=g) + 0.1, logp_ref=(lp + 0.2 * torch.randn(T, generator=g)).float(),
             w_tis=torch.exp(0.1 * torch.randn(T, generator=g)).clamp(max=2.0))
    b["weight"][torch.rand(T, generator=g) < 0.2] = 0.0
    b["weight"][0] = 1.0
    return b


def reference(b, t=1.0, beta=BETA, low=LOW, high=HIGH, grad=True):
    """(loss, dlogits, logp, entropy) in 64 bits, and each row's tolerance of logp."""
    x = b["logits"].to(F64) / t
    T, V = x.shape
    tok = b["tokens"]
    live = (tok >= 0) & (tok < V)
    if grad:
        live &= b["weight"] != 0
    safe = torch.where((tok >= 0) & (tok < V), tok, torch.zeros_like(tok))
    lps = torch.log_softmax(x, dim=1)
    p = lps.exp()
    logp = lps.gather(1, safe[:, None])[:, 0]
    entropy = -torch.where(p > 0, p * lps, torch.zeros_like(p)).sum(dim=1)
    finite = torch.where(torch.isfinite(x), x, x.amax(dim=1, keepdim=True))
    r2 = (finite.amax(dim=1) - finite.amin(dim=1)) * 1.4427
    tol = (180 + 2 * r2) * U + 8 * U * (logp.abs() + finite.abs().amax(dim=1))
    zero = torch.zeros_like(logp)
    out = dict(logp=torch.where(live, logp, zero), entropy=torch.where(live, entropy, zero), tol=tol, r2=r2, live=live)
    if not grad:
        return out
    a, c = b["adv"].to(F64), b["weight"].to(F64)
    w = b["w_tis"].to(F64) if b.get("w_tis") is not None else torch.ones_like(a)
    r = torch.exp(logp - b["logp_old"].to(F64))
    plain, cut = r * a, r.clamp(low, high) * a
    term = -w * torch.minimum(plain, cut)
    slope = torch.where(plain <= cut, -w * plain, zero)
    scale = w * plain.abs()
    if b.get("logp_ref") is not None:
        d = b["logp_ref"].to(F64) - logp
        term = term + beta * (torch.exp(d) - d - 1)
        slope = slope + beta * (1 - torch.exp(d))
        scale = scale + beta * (1 + torch.exp(d) + d.abs())
    k = torch.where(live, c * slope / t, zero)
    dl = -k[:, None] * p
    dl.scatter_add_(1, safe[:, None], torch.where(live, k, zero)[:, None])
    out.update(loss=torch.where(live, c * term, zero).sum(), dlogits=torch.where(live[:, None], dl, torch.zeros_like(dl)),
               # what a rounding of logp may do to a token's term and factor
               dterm=torch.where(live, c * scale * (2 * tol + 16 * U), zero), k=k,
               dk=torch.where(live, c * scale * (2 * tol + 16 * U) / t, zero), p=p, token=safe)
    return out


def on(b):
    return {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in b.items()}


def call(b, t=1.0, beta=BETA, low=LOW, high=HIGH, **kw):
    g = on(b)
    return fp8q.policy_loss(g["logits"], g["tokens"], g["logp_old"], g["adv"], g["weight"], low, high, beta=beta,
                            logp_ref=g.get("logp_ref"), w_tis=g.get("w_tis"), temperature=t, **kw)


def check(got, ref, dtype, what=""):
    loss, dl, logp, entropy = got
    within(logp, ref["logp"], ref["tol"], what + " logp")
    within(entropy, ref["entropy"], 4 * (1 + ref["r2"]) * ref["tol"], what + " entropy")
    # the terms, then a sum of T roundings of the whole in the final conversion
    within(loss, ref["loss"].reshape(1), float(ref["dterm"].sum() + 2 * U * abs(ref["loss"])) + 1e-30, what + " loss")
    rel = (2 * ref["tol"] + 2.0 ** -22 + 2 * U * ref["r2"])[:, None]
    p = ref["p"].clone()
    p.scatter_(1, ref["token"][:, None], 1.0)  # (delta - p: at the token |k| itself bounds what is lost)
    bound = (ref["k"].abs()[:, None] * rel + ref["dk"][:, None]) * p
    whole = ref["dlogits"].abs() + bound
    bound = bound + (bf16_half(whole) if dtype == torch.bfloat16 else U * whole) + 1e-38
    within(dl, ref["dlogits"], bound, what + " dlogits")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_loss(shape, dtype):
    T, V = shape
    t = 0.7 if V % 2 else 1.0
    print("policy loss", shape, dtype, flush=True)
    b = batch(T, V, dtype, seed=31, t=t)
    ref = reference(b, t=t)
    got = call(b, t=t)
    check(got, ref, dtype)
    for a, c, n in zip(got, call(b, t=t), ("loss", "dlogits", "logp", "entropy")):
        same(a, c, n + " of two runs")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES + [(129, 131072), (1000, 4097)])
def test_logprobs(shape, dtype):
    T, V = shape
    b = batch(T, V, dtype, seed=32)
    b["tokens"][T // 2] = -100 if T > 1 else 0
    ref = reference(b, grad=False)
    logp, entropy = fp8q.token_logprobs(b["logits"].to(DEV), b["tokens"].to(DEV))
    within(logp, ref["logp"], ref["tol"], "logp")
    within(entropy, ref["entropy"], 4 * (1 + ref["r2"]) * ref["tol"], "entropy")


@pytest.mark.parametrize("T,V", [(40, 1000), (9, 60000), (130, 33000)])
def test_rows_that_do_not_count(T, V):
    """Rows of weight 0 and of tokens outside the vocabulary hold NaN and
    infinities: nothing of them shows, their gradients are zeros; and batches of
    nothing else."""
    b = batch(T, V, torch.bfloat16, seed=33)
    b["tokens"][1], b["tokens"][2], b["tokens"][3] = -100, V, -(1 << 40)
    b["weight"][4:6] = 0.0
    ref = reference(b)
    b["logits"][1], b["logits"][2, 5], b["logits"][4] = float("nan"), float("inf"), float("-inf")
    b["logits"][5], b["logp_old"][5], b["adv"][5] = float("nan"), float("nan"), float("inf")
    got = call(b)
    check(got, ref, torch.bfloat16)
    assert not bool((got[1].cpu()[1:6][torch.tensor([0, 1, 2, 3, 4])] != 0).any())
    b["weight"][:] = 0.0
    loss, dl, logp, entropy = call(b)
    assert float(loss) == 0.0 and not bool(dl.any()) and not bool(logp.any()) and not bool(entropy.any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(20, 999), (5, 70001), (130, 40000)])
def test_masked_logits(T, V, dtype):
    """Logits of -inf (a restricted vocabulary) and of the type's lowest value
    have probability and gradient 0; a row of nothing but -inf, NaN or +inf gives
    NaN, and no other row does."""
    b = batch(T, V, dtype, seed=34)
    b["logits"][:, V // 3:] = float("-inf")
    b["logits"][1, : V // 3] = torch.finfo(dtype).min
    b["logits"][1, 3] = 0.5
    b["tokens"] %= V // 3
    b["tokens"][1] = 3
    b["weight"][:] = 1.0
    b["logp_old"][1] = b["logp_ref"][1] = 0.0  # (its token has probability 1)
    ref = reference(b)
    ref["tol"][1], ref["r2"][1] = 1e-6, 0.0
    got = call(b)
    dl = got[1].cpu()
    assert not bool(dl[:, V // 3:].any())
    within(got[2], ref["logp"], ref["tol"], "logp")
    within(got[3], ref["entropy"], 4 * (1 + ref["r2"]) * ref["tol"], "entropy")
    b["logits"][2] = float("-inf")
    b["logits"][3, 4] = float("nan")
    b["logits"][4, 5] = float("inf")
    _, dl, logp, entropy = call(b)
    bad = torch.tensor([i in (2, 3, 4) for i in range(T)])
    assert torch.equal(torch.isnan(logp.cpu()), bad) and torch.equal(torch.isnan(entropy.cpu()), bad)
    assert torch.equal(torch.isnan(dl.cpu().float()).any(dim=1), bad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(20, 999), (5, 70001), (130, 40000)])
def test_logits_at_the_ends_of_the_range(T, V, dtype):
    """Rows of nothing but the type's lowest value (a mask that leaves nothing),
    or its largest, are uniform; the largest among others takes everything; rows
    beside them keep their results."""
    b = batch(T, V, dtype, seed=43)
    want = call(b, t=0.5)
    top = torch.finfo(dtype).max
    b["logits"][1], b["logits"][2], b["logits"][3] = -top, top, -top
    b["logits"][3, 5] = top
    b["tokens"][3] = 5
    b["weight"][1:4] = 1.0
    b["logp_old"][1:3] = b["logp_ref"][1:3] = -math.log(V)
    b["logp_old"][3] = b["logp_ref"][3] = 0.0
    ref = reference(b, t=0.5)
    ref["tol"][1:4], ref["r2"][1:4] = 1e-5, 0.0
    loss, dl, logp, entropy = call(b, t=0.5)
    within(logp, ref["logp"], ref["tol"], "logp")
    within(entropy, ref["entropy"], 4 * (1 + ref["r2"]) * ref["tol"], "entropy")
    d = dl.cpu().to(F64)[1:4]
    half = bf16_half(ref["dlogits"][1:4]) if dtype == torch.bfloat16 else 0.0
    assert bool(((d - ref["dlogits"][1:4]).abs() <= 1e-4 * ref["dlogits"][1:4].abs() + half + 1e-30).all())
    for i in range(T):
        if not 1 <= i < 4:
            same(dl[i], want[1][i], "row %d" % i)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(24, 999), (12, 70001), (130, 40000)])
def test_large_logits(T, V, dtype):
    """Rows far from 0, up to where a logit times log2(e) / t leaves fp32's range:
    a common offset of the logits costs no accuracy (the fp32 exponent is relative
    to the row's maximum), and of logits far apart the largest takes everything.
    With an offset of 2^28 / t the fp32 exponents are up to 2^4 from the maximum's,
    so a log-probability is good to 2^-24 of some 2^5, below 1e-5."""
    b = batch(T, V, dtype, seed=47)
    gen = torch.Generator().manual_seed(48)
    rows = 0
    for offset in (2.0**12, -(2.0**20), 2.0**24, -(2.0**27), 3e12, -1e37):
        b["logits"][rows] = (offset + 4 * torch.randn(V, generator=gen, dtype=F64)).to(dtype).to(b["logits"].device)
        rows += 1
    for scale in (1e9, 1e12, 1e20, 4e37):
        b["logits"][rows] = (scale * torch.randn(V, generator=gen, dtype=F64)).to(dtype).to(b["logits"].device)
        b["tokens"][rows] = b["logits"][rows].argmax().to(b["tokens"].dtype)
        rows += 1
    b["weight"][:rows] = 1.0
    logp = reference(b, t=0.5)["logp"][:rows].float()
    b["logp_old"][:rows] = logp.to(b["logp_old"].device)
    b["logp_ref"][:rows] = logp.to(b["logp_ref"].device)
    ref = reference(b, t=0.5)
    ref["tol"][:rows], ref["r2"][:rows] = 1e-5 + 2.0**-22 * ref["logp"][:rows].abs(), 0.0
    loss, dl, logp, entropy = call(b, t=0.5)
    within(logp, ref["logp"], ref["tol"], "logp")
    within(entropy, ref["entropy"], 4 * (1 + ref["r2"]) * ref["tol"], "entropy")
    assert math.isfinite(float(loss))
    d = dl.cpu().to(F64)[:rows]
    want = ref["dlogits"][:rows]
    half = bf16_half(want) if dtype == torch.bfloat16 else 0.0
    assert bool(((d - want).abs() <= 1e-4 * want.abs() + half + 1e-9 * want.abs().amax(dim=1, keepdim=True)).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(33, 1000), (6, 65537), (135, 20000)])
def test_layouts(T, V, dtype):
    """Rows that start at any element (a slice of a wider buffer), gradients of
    another alignment, in place, on a stream of its own, a given workspace."""
    b = batch(T, V, dtype, seed=35)
    want = call(b)
    for first in (0, 1, 3):
        wide = torch.full((T, V + 5), float("nan"), dtype=dtype, device=DEV)
        x = wide[:, first:first + V]
        x.copy_(b["logits"])
        g = on(b)
        args = (g["tokens"], g["logp_old"], g["adv"], g["weight"], LOW, HIGH)
        kw = dict(beta=BETA, logp_ref=g["logp_ref"], w_tis=g["w_tis"])
        ws = torch.full((fp8q.lib().fp8q_policy_loss_workspace(T, V),), 0xff, dtype=torch.uint8, device=DEV)
        dl = torch.full((T, V + 3), 3.0, dtype=dtype, device=DEV)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            got = fp8q.policy_loss(x, *args, **kw, dlogits=dl[:, 2:2 + V], workspace=ws)
            lp = fp8q.token_logprobs(x, g["tokens"], workspace=ws)
        torch.cuda.synchronize()
        live = (b["weight"] != 0).to(DEV)
        # (another alignment sums in another order)
        for i, tol in ((0, 2e-5), (2, 2e-5), (3, 2e-4)):
            assert torch.allclose(got[i], want[i], rtol=2e-5, atol=tol), i
        assert torch.allclose(got[1].float(), want[1].float(), rtol=1e-2, atol=1e-7 * float(want[1].float().abs().max()))
        assert torch.allclose(lp[0][live], got[2][live], rtol=2e-5, atol=2e-5)
        assert bool((dl[:, :2] == 3).all()) and bool((dl[:, 2 + V:] == 3).all())
        place = fp8q.policy_loss(x, *args, **kw, dlogits=x)
        assert place[1] is x
        ref = fp8q.policy_loss(wide[:, first:first + V].copy_(b["logits"]), *args, **kw)
        same(place[0], ref[0], "loss in place")
        wide[:, first:first + V].copy_(b["logits"])
        same(fp8q.policy_loss(x, *args, **kw, dlogits=x)[1], ref[1], "gradient in place")


def test_optional_terms_and_device_bounds():
    """Without reference and importance weights; and with the bounds that
    Calibrated Clipping left on the device."""
    b = batch(50, 3000, torch.float32, seed=36)
    plain = {k: v for k, v in b.items() if k not in ("logp_ref", "w_tis")}
    check(call(plain, beta=0.3), reference(plain, beta=0.3), torch.float32, "plain")
    clip = torch.zeros(80, dtype=torch.uint8)
    clip[:16] = torch.tensor([0.91, 1.05], dtype=F64).view(torch.uint8)  # l_new, h_new
    ref = reference(b, low=float(torch.tensor(0.91, dtype=torch.float32)), high=float(torch.tensor(1.05)))
    got = call(b, low=0.0, high=0.0, clip=clip.to(DEV))
    check(got, ref, torch.float32, "device bounds")


def test_every_branch_of_the_clip():
    """Both signs of the advantage on both sides of both bounds, and an advantage
    of 0: the gradient is cut exactly where the smaller side is the clipped one."""
    T, V = 14, 64
    b = batch(T, V, torch.float32, seed=37)
    lp = torch.log_softmax(b["logits"].to(F64), dim=1).gather(1, b["tokens"][:, None])[:, 0]
    r = torch.tensor([0.5, 0.9, 1.1, 1.5, 0.79, 0.81, 1.23, 1.25, 0.5, 1.5, 1e-3, 50.0, 1.0, 1.0], dtype=F64)
    b["logp_old"] = (lp - r.log()).float()
    b["adv"] = torch.tensor([1.0, 1, 1, 1, -1, -1, 1, 1, -1, -1, -1, 1, 0, -2])
    b["weight"][:] = 0.25
    del b["logp_ref"]
    ref = reference(b)
    assert [bool(k == 0) for k in ref["k"]] == [False, False, False, True, True, False, False, True, True, False, True,
                                               True, True, False]
    check(call(b), ref, torch.float32)


@pytest.mark.parametrize("T,V", [(9, 900), (9, 70001), (130, 900)])
def test_ratios_past_the_range(T, V):
    """exp(logp - logp_old) and exp(logp_ref - logp) past fp32: an advantage, an
    importance weight or a KL coefficient of zero makes nothing of them, a clipped
    ratio is cut as ever, and what has no finite value in fp32 is infinite."""
    b = batch(T, V, torch.float32, seed=49)
    b["weight"][:] = 0.5
    b["logp_old"][:4] = -400.0
    b["adv"][:4] = torch.tensor([0.0, 2.0, -2.0, 0.5])
    b["w_tis"][2] = 0.0
    b["logp_ref"][:4] = 400.0
    ref = reference({k: v for k, v in b.items() if k != "logp_ref"}, beta=0.0)
    check(call(b, beta=0.0), ref, torch.float32)
    assert not bool(ref["dlogits"][:4].any())
    b["w_tis"][2] = 1.0
    loss, _, logp, _ = call(b, beta=0.0)
    assert float(loss) == math.inf
    within(logp, ref["logp"], ref["tol"], "logp")


def test_gradient_against_differences():
    """The gradient along random directions against central differences of the
    64-bit loss."""
    b = batch(12, 300, torch.float32, seed=38, t=0.8)
    _, dl, _, _ = call(b, t=0.8)
    u = torch.randn(12, 300, generator=torch.Generator().manual_seed(39), dtype=F64)
    e = 1e-5
    sides = []
    for s in (e, -e):
        c = dict(b, logits=b["logits"].to(F64) + s * u)
        sides.append(float(reference(c, t=0.8)["loss"]))
    along = (sides[0] - sides[1]) / (2 * e)
    got = dl.cpu().to(F64) * u
    assert abs(float(got.sum()) - along) <= 1e-5 * float(got.abs().sum()) + 1e-8


def test_offsets_past_32_bits():
    """Rows that start past 2^31 elements, and a gradient of that size."""
    V, ld = 1000, 1 << 24
    b = batch(150, V, torch.bfloat16, seed=40)
    want = call(b)
    far = torch.empty(150 * ld, dtype=torch.bfloat16, device=DEV).view(150, ld)[:, :V]
    far.copy_(b["logits"])
    g = on(b)
    got = fp8q.policy_loss(far, g["tokens"], g["logp_old"], g["adv"], g["weight"], LOW, HIGH, beta=BETA,
                           logp_ref=g["logp_ref"], w_tis=g["w_tis"], dlogits=far)
    for a, c, n in zip(got, want, ("loss", "dlogits", "logp", "entropy")):
        same(a, c, n)


def test_graph_replay():
    """Captured once, replayed with the program's own work between: every replay
    equals the call."""
    b = on(batch(40, 70001, torch.bfloat16, seed=41))
    ws = torch.empty(fp8q.lib().fp8q_policy_loss_workspace(40, 70001), dtype=torch.uint8, device=DEV)
    out = dict(loss=torch.empty(1, device=DEV), dlogits=torch.empty_like(b["logits"]), logp=torch.empty(40, device=DEV),
               entropy=torch.empty(40, device=DEV), workspace=ws)
    args = (b["logits"], b["tokens"], b["logp_old"], b["adv"], b["weight"], LOW, HIGH)
    want = fp8q.policy_loss(*args, beta=BETA, logp_ref=b["logp_ref"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fp8q.policy_loss(*args, beta=BETA, logp_ref=b["logp_ref"], **out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            fp8q.policy_loss(*args, beta=BETA, logp_ref=b["logp_ref"], **out)
    for i in range(3):
        for t in (out["loss"], out["dlogits"], out["logp"], out["entropy"]):
            t.fill_(float("nan"))
        ws.fill_(0xff)
        torch.randn(1000, 1000, device=DEV).sum()
        graph.replay()
        torch.cuda.synchronize()
        for a, c, n in zip((out["loss"], out["dlogits"], out["logp"], out["entropy"]), want,
                           ("loss", "dlogits", "logp", "entropy")):
            same(a, c, "%s of replay %d" % (n, i))


def test_refusals():
    b = on(batch(8, 200, torch.bfloat16, seed=42))
    x, args = b["logits"], (b["tokens"], b["logp_old"], b["adv"], b["weight"], LOW, HIGH)
    f = fp8q.policy_loss
    for bad in (lambda: f(x.half(), *args), lambda: f(x[0], *args), lambda: f(x, args[0].int(), *args[1:]),
                lambda: f(x, args[0][:4], *args[1:]), lambda: f(x, args[0], args[1].double(), *args[2:]),
                lambda: f(x, *args, w_tis=b["adv"][:3]), lambda: f(x, *args, dlogits=x.float()),
                lambda: f(x, *args, workspace=torch.empty(8, dtype=torch.uint8, device=DEV)),
                lambda: f(x.t(), *args), lambda: fp8q.token_logprobs(x.cpu(), b["tokens"]),
                lambda: f(x, *args, clip=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(x, *args, temperature=0.0), lambda: f(x, *args, temperature=float("nan")),
                lambda: f(x, *args[:4], 1.2, 0.8), lambda: f(x, *args[:4], float("nan"), 1.2),
                lambda: f(x, *args, beta=float("nan")), lambda: fp8q.token_logprobs(x, b["tokens"], temperature=-1.0)):
        with pytest.raises(fp8q.Fp8qError) as e:
            bad()
        assert e.value.status == -1
