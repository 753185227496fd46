"""Nothing is written past what a call owns: workspaces, vectors and rows with guards behind
them; the sort's sizes at which another kernel takes over, and tokens that all fall into one of
its classes; the large sort captured into a graph."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, same
from test_gpu_zb_embedding import BF16, check_gradient

pytestmark = pytest.mark.gpu

GUARD = 0x5A


def guarded(n, dtype=torch.uint8):
    """A vector of n elements, and a check that nothing behind it has changed."""
    size = torch.empty(0, dtype=dtype).element_size()
    raw = torch.full((n * size + 4096,), GUARD, dtype=torch.uint8, device=DEV)
    return raw[:n * size].view(dtype), lambda: bool((raw[n * size:] == GUARD).all())


@pytest.mark.parametrize("T", [1, 64, 256, 257, 1024, 4096, 4097, 8192, 8193, 16384, 16385])
@pytest.mark.parametrize("step", [1, 64])
def test_gradient_where_the_sort_changes(T, step):
    """step 64: all tokens in one class, with as many keys in it as it can have."""
    V, C = 64 * 700, 32
    print("embedding gradient", T, step, flush=True)
    g = torch.Generator().manual_seed(T)
    t = torch.randint(0, V // step, (T,), generator=g) * step
    t[torch.rand(T, generator=g) < 0.05] = -1
    dy = torch.randn(T, C, generator=g).bfloat16()
    for dtype in (torch.float32, BF16):
        need = fp8q.lib().fp8q_embedding_backward_workspace(T, V, C)
        ws, intact = guarded(need)
        flat, table_intact = guarded(V * (C + 8), dtype)
        flat.fill_(9.0)
        dw = flat.view(V, C + 8)[:, :C]
        got = fp8q.embedding_backward(dy.to(DEV), t.to(DEV), V, 0.5, dtype=dtype, dweight=dw, workspace=ws)
        assert got is dw and intact() and table_intact() and bool((flat.view(V, C + 8)[:, C:] == 9.0).all())
        check_gradient(dw.contiguous(), dy, t, V, 0.5, dtype, what="%s" % dtype)


def test_large_sort_captured():
    T, V, C = 20000, 3000, 64
    g = torch.Generator(device=DEV).manual_seed(11)
    t, dy = torch.empty(T, dtype=torch.int64, device=DEV), torch.randn(T, C, generator=g, device=DEV).bfloat16()
    t.fill_(1)
    dw = torch.empty(V, C, device=DEV)
    ws = torch.empty(fp8q.lib().fp8q_embedding_backward_workspace(T, V, C), dtype=torch.uint8, device=DEV)

    def step():
        fp8q.embedding_backward(dy, t, V, dweight=dw, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        t.copy_(torch.randint(-1, V + 1, (T,), generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = dw.clone()
        step()
        same(got, dw, "replay %d" % i)


@pytest.mark.parametrize("T,V,k", [(3, 90000, 20), (64, 131072, 64), (200, 700, 5), (1, 1, 1), (9, 64, 64)])
def test_alternatives(T, V, k):
    g = torch.Generator().manual_seed(12)
    x = torch.randn(T, V, generator=g).bfloat16().to(DEV)
    tokens = torch.randint(-1, V, (T,), generator=g).to(DEV)
    need = fp8q.lib().fp8q_top_logprobs_workspace(T, V, k)
    logp, entropy, ids, top, ws = (guarded(n, d) for n, d in ((T, torch.float32), (T, torch.float32), (T * k, torch.int64),
                                                              (T * k, torch.float32), (max(need, 16), torch.uint8)))
    got = fp8q.top_logprobs(x, tokens, k, logp=logp[0], entropy=entropy[0], ids=ids[0].view(T, k), top=top[0].view(T, k),
                            workspace=ws[0])
    assert all(o[1]() for o in (logp, entropy, ids, top, ws))
    for a, b in zip(got, fp8q.top_logprobs(x, tokens, k)):
        same(a, b, "given outputs")


@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 31), (33, 257), (40, 1000), (2000, 513)])
def test_quantized(rows, cols):
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(13)).bfloat16().to(DEV)
    want = fp8q.quantize_mx4(x)
    codes, scales, y = guarded(want[0].numel()), guarded(want[1].numel()), guarded(rows * cols, BF16)
    got = fp8q.quantize_mx4(x, codes=codes[0].view_as(want[0]), scales=scales[0])
    fp8q.dequantize_mx4(*got, cols, out=y[0].view(rows, cols))
    assert codes[1]() and scales[1]() and y[1]()
    for a, b in zip(got, want):
        same(a, b, "given outputs")
    same(y[0].view(rows, cols), fp8q.dequantize_mx4(*want, cols), "values")


@pytest.mark.parametrize("T", [300, 5000])
def test_vocabulary_too_large_for_the_small_sort(T):
    V, C = (1 << 21) + 64, 16
    print("embedding gradient", T, V, flush=True)
    g = torch.Generator().manual_seed(T)
    t = torch.randint(V - 400, V + 20, (T,), generator=g)
    t[::7] = torch.randint(0, V, (t[::7].numel(),), generator=g)
    dy = torch.randn(T, C, generator=g).bfloat16()
    got = fp8q.embedding_backward(dy.to(DEV), t.to(DEV), V, 2.0)
    check_gradient(got, dy, t, V, 2.0, torch.float32, what="large vocabulary")
    old = torch.randn(V, C, generator=g)
    into = fp8q.embedding_backward(dy.to(DEV), t.to(DEV), V, 2.0, dweight=old.to(DEV), accumulate=True)
    check_gradient(into, dy, t, V, 2.0, torch.float32, old=old, what="added")
