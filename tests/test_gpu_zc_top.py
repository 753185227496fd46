"""Log-probabilities with the k most probable alternatives, against 64-bit references: indices equal,
log-probabilities and entropies within the tolerances of the log-probabilities alone (see
test_gpu_v_loss.py; an alternative's log-probability is the token's formula)."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, same, strided, within
from test_gpu_v_loss import U, batch, reference

pytestmark = pytest.mark.gpu


def order(x, k):
    """Indices and values of the k largest of each row, equal ones by index; -1 for -inf."""
    v, i = torch.sort(x.to(F64) + 0.0, dim=1, descending=True, stable=True)
    v, i = v[:, :k], i[:, :k]
    return torch.where(v == float("-inf"), torch.full_like(i, -1), i), v


def check(x, tokens, k, t=1.0, got=None, what=""):
    T, V = x.shape
    got = fp8q.top_logprobs(x.to(DEV), tokens.to(DEV), k, temperature=t) if got is None else got
    logp, entropy, ids, top = (v.cpu() for v in got)
    ref = reference(dict(logits=x, tokens=tokens), t=t, grad=False)
    live = ref["live"]
    within(logp, ref["logp"], ref["tol"], "%s logp" % (what,))
    within(entropy, ref["entropy"], 4 * (1 + ref["r2"]) * ref["tol"], "%s entropy" % (what,))
    want, v = order(x, k)
    want[~live] = -1
    bad = ids != want
    assert not bool(bad.any()), (what, ids[bad][:5], want[bad][:5], int(bad.sum()))
    lp = v / t - torch.logsumexp(x.to(F64) / t, dim=1, keepdim=True)
    lp[~live] = 0.0
    none = lp == float("-inf")
    assert bool((top[none] == float("-inf")).all())
    finite = torch.where(none, torch.zeros_like(lp), lp)
    bound = ref["tol"][:, None] + 8 * U * finite.abs()
    within(torch.where(none, torch.zeros_like(top), top), finite, bound, "%s alternatives" % (what,))
    return got


SHAPES = [(1, 1, 1), (2, 3, 3), (3, 8, 5), (5, 100, 64), (130, 1001, 8), (200, 8191, 20), (130, 9000, 1), (150, 20001, 5),
          (140, 40003, 64), (129, 131072, 20), (128, 150001, 2), (1, 50021, 20), (7, 70001, 64), (64, 131072, 20),
          (2, 300007, 5), (3, 65, 64), (300, 64, 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V,k", SHAPES)
def test_alternatives(T, V, k, dtype):
    print("top", T, V, k, dtype, flush=True)
    b = batch(T, V, dtype, seed=41)
    if T > 1:
        b["tokens"][T // 2] = -100
    t = 0.7 if V % 2 else 1.0
    got = check(b["logits"], b["tokens"], k, t)
    for a, c in zip(got, fp8q.top_logprobs(b["logits"].to(DEV), b["tokens"].to(DEV), k, temperature=t)):
        same(a, c, "two runs")


ROWS = [(140, 5000), (140, 20000), (130, 70001), (9, 70001), (2, 200003)]


@pytest.mark.parametrize("T,V", ROWS)
def test_rows_with_structure(T, V):
    """Equal logits (all, but for a few, in a few values), rows in order, one piece of 64 much larger, few
    finite ones, signed zeros: where bounds and room for candidates can go wrong."""
    x = torch.zeros(T, V, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(5)
    n = torch.arange(V)
    kinds = [torch.zeros(V), (n == V - 1).float() + 2.0 * (n == 17), (n % 3).float(), -n / 7.0, n / 5.0,
             10.0 * ((n // 8) % 64 == 5) + torch.randn(V, generator=g), 10.0 * ((n // 4) % 256 == 7) + 0.01 * (n % 97),
             torch.where(n % (V // 3) == 5, 1.0, float("-inf")), torch.where(n == V // 2, -3.0, float("-inf")),
             torch.where(n % 2 == 0, 0.0, -0.0), torch.full((V,), -3.0e38), torch.randint(0, 4, (V,), generator=g).float()]
    for r in range(T):
        x[r] = kinds[r % len(kinds)].bfloat16()
    tokens = torch.where(torch.isinf(x), torch.full_like(x, -1), torch.ones_like(x)).argmax(dim=1)
    for k in (1, 20, 64):
        want, _ = order(x, k)
        logp, entropy, ids, top = (v.cpu() for v in fp8q.top_logprobs(x.to(DEV), tokens.to(DEV), k))
        bad = ids != want
        assert not bool(bad.any()), (k, torch.nonzero(bad)[:5], ids[bad][:5], want[bad][:5])
        # (the same formula for the same logit)
        mine = x.gather(1, tokens[:, None]) == x.gather(1, want.clamp(min=0))
        mine &= want >= 0
        assert bool((top == logp[:, None])[mine].all())
        both, ent = fp8q.token_logprobs(x.to(DEV), tokens.to(DEV))
        scale = x.float().abs().where(torch.isfinite(x.float()), torch.zeros(1)).amax(dim=1).to(F64)
        within(logp, both.cpu().to(F64), 2 * (180 + 20 * scale) * U, "as the log-probabilities alone")


@pytest.mark.parametrize("T,V", [(140, 4000), (9, 60000)])
def test_rows_that_hold_no_numbers(T, V):
    """NaN, +inf or nothing but -inf in a row: NaN there, indices in range or -1; the others as ever.  A row of
    padding is not read."""
    b = batch(T, V, torch.float32, seed=42)
    x, tok = b["logits"], b["tokens"]
    want = check(x, tok, 7)
    x[1, 5], x[2, 9], x[3], x[4] = float("nan"), float("inf"), float("-inf"), float("nan")
    tok[5] = -1
    x[5] = float("nan")
    got = fp8q.top_logprobs(x.to(DEV), tok.to(DEV), 7)
    for a, c in zip(got, want):
        same(torch.cat((a[:1], a[6:])), torch.cat((c[:1], c[6:])), "the other rows")
    logp, entropy, ids, top = (v.cpu() for v in got)
    assert bool(torch.isnan(logp[1:5]).all()) and bool(torch.isnan(entropy[1:5]).all())
    assert bool(((ids[1:5] >= -1) & (ids[1:5] < V)).all()) and ids[2, 0] == 9 and bool((ids[3:6] == -1).all())
    assert bool((ids[1] != 5).all())
    assert float(logp[5]) == 0.0 and float(entropy[5]) == 0.0 and bool((top[5] == 0.0).all())


def test_unaligned_rows_given_outputs_and_stream():
    b = batch(40, 5001, torch.bfloat16, seed=43)
    want = [v.clone() for v in fp8q.top_logprobs(b["logits"].to(DEV), b["tokens"].to(DEV), 9)]
    s = torch.cuda.Stream()
    x = strided(b["logits"].to(DEV), 1)
    tokens = b["tokens"].to(DEV)
    T = 40
    out = dict(logp=torch.empty(T, device=DEV), entropy=torch.empty(T, device=DEV),
               ids=torch.empty(T, 9, dtype=torch.int64, device=DEV), top=torch.empty(T, 9, device=DEV))
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = fp8q.top_logprobs(x, tokens, 9, **out)
    s.synchronize()
    assert got[2] is out["ids"] and got[0] is out["logp"]
    assert bool((got[2] == want[2]).all())
    check(b["logits"], b["tokens"], 9, got=got)


@pytest.mark.parametrize("T,V", [(4, 90000), (200, 3000)])
def test_captured_and_replayed(T, V):
    g = torch.Generator(device=DEV).manual_seed(11)
    x = torch.randn(T, V, generator=g, device=DEV).bfloat16()
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV)
    fp8q.top_logprobs(x, tokens, 5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fp8q.top_logprobs(x, tokens, 5)
    for i in range(4):
        x.copy_(3.0 * torch.randn(T, V, generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(out, fp8q.top_logprobs(x, tokens, 5)):
            same(a, c, "replay %d" % i)
