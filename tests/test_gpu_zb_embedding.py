"""Embedding rows and the table's gradient.

A looked-up row is one fp32 product and its rounding to bf16, compared bit for bit.  A gradient's
row of n terms is summed in fp32 (at most n roundings of a partial sum, which is at most sum |dy|),
times scale (one more), added to what is there (one more), and rounded to its type: |dw - ref| <=
(n + 1) 2^-24 |scale| sum |dy| + 2^-24 |result| + half a unit of its type."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, F64, bf16_half, same, strided, within

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def tokens_of(T, V, seed, padding=0.1):
    g = torch.Generator().manual_seed(seed)
    t = (torch.exp(torch.rand(T, generator=g, dtype=F64) * torch.log(torch.tensor(float(V + 1)))).long() - 1).clamp(0, V - 1)
    outside = torch.tensor([-1, V, -100, 1 << 40])[torch.randint(0, 4, (T,), generator=g)]
    return torch.where(torch.rand(T, generator=g) < padding, outside, t)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,C", [(1, 1, 16), (3, 7, 48), (8, 1000, 4096), (130, 500, 2064), (1001, 3000, 80),
                                   (4097, 50, 512)])
def test_rows(T, V, C, dtype):
    g = torch.Generator().manual_seed(T)
    w = torch.randn(V, C, generator=g).to(dtype)
    t = tokens_of(T, V, T + 1)
    live = (t >= 0) & (t < V)
    for scale in (1.0, 45.254833995939045, -0.3):
        want = (w[t.clamp(0, V - 1)].float() * torch.tensor(scale, dtype=F32)).bfloat16()
        want = torch.where(live[:, None], want, torch.zeros_like(want))
        same(fp8q.embedding(w.to(DEV), t.to(DEV), scale), want, (T, V, C, scale))
    wide = torch.full((T, C + 24), 9.0, dtype=BF16, device=DEV)
    got = fp8q.embedding(strided(w.to(DEV), 8), t.to(DEV), -0.3, out=wide[:, :C])
    same(got, want, "strided")
    assert bool((wide[:, C:] == 9.0).all())


def check_gradient(got, dy, t, V, scale, dtype, old=None, what=""):
    T, C = dy.shape
    live = (t >= 0) & (t < V)
    n = torch.bincount(t[live], minlength=V).to(F64)
    ref, absum = torch.zeros(V, C, dtype=F64), torch.zeros(V, C, dtype=F64)
    ref.index_add_(0, t[live], dy[live].to(F64))
    absum.index_add_(0, t[live], dy[live].to(F64).abs())
    s = float(torch.tensor(scale, dtype=F32))
    ref = ref * s
    bound = (n + 1)[:, None] * U * abs(s) * absum
    if old is not None:
        ref = ref + torch.where(n[:, None] > 0, old.to(F64), torch.zeros_like(ref))
        bound = bound + U * (ref.abs() + bound)
    whole = ref.abs() + bound
    bound = bound + (bf16_half(whole) if dtype is BF16 else U * whole) + 2.0 ** -149
    used = n > 0
    if bool(used.any()):
        within(got.cpu()[used], ref[used], bound[used], what)
    rest = torch.zeros(V, C, dtype=dtype) if old is None else old
    same(got.cpu()[~used], rest[~used], "rows of no token")


# one chunk and many, runs across chunks, the sort's workgroup full, and more tokens than it takes
CASES = [(1, 1, 16), (1, 40, 4096), (31, 5, 16), (32, 3, 48), (33, 1, 2048), (64, 4, 2064), (100, 100000, 32),
         (1000, 7, 96), (1023, 3000, 256), (5003, 32000, 64), (16384, 999, 32), (16385, 999, 32), (40000, 20001, 16),
         (70000, 3, 32), (200, 300000, 16), (20000, 1 << 20, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,C", CASES)
def test_gradient(T, V, C, dtype):
    print("embedding gradient", T, V, C, dtype, flush=True)
    g = torch.Generator().manual_seed(T + V)
    dy = torch.randn(T, C, generator=g).bfloat16()
    t = tokens_of(T, V, T + 2)
    scale = 1.0 if T % 2 else 11.3
    d, tk = dy.to(DEV), t.to(DEV)
    got = fp8q.embedding_backward(d, tk, V, scale, dtype=dtype)
    check_gradient(got, dy, t, V, scale, dtype, what=(T, V, C))
    need = fp8q.lib().fp8q_embedding_backward_workspace(T, V, C)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    again = fp8q.embedding_backward(d, tk, V, scale, dtype=dtype, workspace=ws,
                                    dweight=torch.full((V, C), float("nan"), dtype=dtype, device=DEV))
    same(again, got, "two runs, another workspace")
    # added to what is there; rows of no token keep what they hold, NaN too
    old = torch.randn(V, C, generator=g).to(dtype)
    n = torch.bincount(t[(t >= 0) & (t < V)], minlength=V)
    old[n == 0] = float("nan")
    wide = strided(old.to(DEV), 8)
    into = fp8q.embedding_backward(d, tk, V, scale, dtype=dtype, dweight=wide, accumulate=True, workspace=ws)
    check_gradient(into, dy, t, V, scale, dtype, old=old, what="accumulated")


@pytest.mark.parametrize("T", [1, 33, 5000, 17000])
def test_one_token_and_none(T):
    g = torch.Generator().manual_seed(T)
    dy = torch.randn(T, 64, generator=g).bfloat16()
    for value, V in ((0, 1), (4, 5), (-1, 5), (5, 5)):
        t = torch.full((T,), value)
        got = fp8q.embedding_backward(dy.to(DEV), t.to(DEV), V)
        check_gradient(got, dy, t, V, 1.0, F32, what=value)


def test_padding_is_not_read():
    t = torch.tensor([3, -1, 3, 9, 0])
    dy = torch.randn(5, 32).bfloat16()
    got = fp8q.embedding_backward(dy.to(DEV), t.to(DEV), 9)
    dy[1], dy[3] = float("nan"), float("inf")
    same(fp8q.embedding_backward(strided(dy.to(DEV), 16), t.to(DEV), 9), got, "rows of padding")


def test_differences():
    """The gradient against differences of sum(dy * embedding(w)) in the table's entries."""
    g = torch.Generator().manual_seed(8)
    T, V, C, scale = 40, 6, 16, 3.0
    w, dy = torch.randn(V, C, generator=g), torch.randn(T, C, generator=g).bfloat16()
    t = tokens_of(T, V, 9)
    got = fp8q.embedding_backward(dy.to(DEV), t.to(DEV), V, scale).cpu().to(F64)

    def loss(w):
        # (the embedding's rounding to bf16 is not differentiated)
        live = ((t >= 0) & (t < V)).to(F64)[:, None]
        return float((dy.to(F64) * live * scale * w.to(F64)[t.clamp(0, V - 1)]).sum())

    for v, c in ((0, 0), (1, 15), (V - 1, 7)):
        h = 2.0 ** -10
        up, down = w.to(F64).clone(), w.to(F64).clone()
        up[v, c] += h
        down[v, c] -= h
        n = int((t == v).sum())
        # (linear: the difference is off by the roundings of two sums in 64 bits alone)
        assert abs((loss(up) - loss(down)) / (2 * h) - float(got[v, c])) <= (n + 2) * U * scale * float(
            dy[t == v].abs().sum()) + 1e-9


def test_captured_and_replayed():
    """A captured step (rows, then the gradient added twice into one table) gives, at every replay, what the
    calls give one by one, with other eager calls and synchronizations in between."""
    g = torch.Generator(device=DEV).manual_seed(10)
    T, V, C = 3000, 700, 128
    w = torch.randn(V, C, generator=g, device=DEV).bfloat16()
    t = torch.randint(-1, V + 1, (T,), generator=g, device=DEV)
    dy = torch.randn(T, C, generator=g, device=DEV).bfloat16()
    out, dw = torch.empty(T, C, dtype=BF16, device=DEV), torch.empty(V, C, device=DEV)
    ws = torch.empty(fp8q.lib().fp8q_embedding_backward_workspace(T, V, C), dtype=torch.uint8, device=DEV)

    def step():
        fp8q.embedding(w, t, 2.0, out=out)
        fp8q.embedding_backward(dy, t, V, 2.0, dweight=dw, workspace=ws)
        fp8q.embedding_backward(dy, t, V, 2.0, dweight=dw, accumulate=True, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        t.copy_(torch.randint(-1, V + 1, (T,), generator=g, device=DEV))
        dy.copy_(torch.randn(T, C, generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), dw.clone()
        step()
        same(got[0], out, "rows, replay %d" % i)
        same(got[1], dw, "gradient, replay %d" % i)
