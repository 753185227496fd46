"""The sorted gradient (more than 256 tokens), where test_gpu_ze_far.py and test_gpu_zb_embedding.py have fewer:
rows of dy and of the table whose offsets pass 32 bits, padding that is not read, a table of just under 2^33
elements, and, with the alternatives of split rows, workspaces on two streams at once."""
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, same
from test_gpu_zb_embedding import check_gradient, tokens_of
from test_gpu_ze_far import FAR, far, rand

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# tokens of the small sort, of its most rounds, and of the large one
SORTED = [300, 9001, 17000]


@pytest.mark.parametrize("T", [5] + SORTED)
@pytest.mark.parametrize("accumulate", [False, True])
def test_padding_is_not_read(T, accumulate):
    """NaN and infinities in the rows of padding, in every part of a chunk and at both ends."""
    print("padding", T, accumulate, flush=True)
    V, C = 97, 48
    t = tokens_of(T, V, T + 31, padding=0.3)
    t[0], t[-1] = -1, V
    outside = (t < 0) | (t >= V)
    dy = rand(T, C, seed=T)
    old = rand(V, C, F32, seed=T + 1)

    def call(dy):
        into = old.clone()
        return fp8q.embedding_backward(dy, t.to(DEV), V, 0.5, dweight=into, accumulate=accumulate)

    got = call(dy)
    bad = dy.clone()
    bad[outside.to(DEV)] = float("nan")
    bad[int(torch.nonzero(outside)[-1])] = float("inf")
    same(call(bad), got, "rows of padding")
    check_gradient(got, dy.cpu(), t, V, 0.5, F32, old=old.cpu() if accumulate else None, what=T)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", SORTED)
def test_far_rows_of_dy(T, dtype):
    """The last row starts 2^32 elements and more from the first."""
    V, C = 53, 96
    ld = -(-((1 << 32) + (1 << 28)) // (T - 1)) // 8 * 8
    print("far dy", T, dtype, ld, flush=True)
    assert (T - 1) * ld > 1 << 32
    dy, t = rand(T, C, seed=T + 2), tokens_of(T, V, T + 32).to(DEV)
    t[-3:] = torch.tensor([V - 1, 0, V - 1], device=DEV)
    want = fp8q.embedding_backward(dy, t, V, 1.5, dtype=dtype)
    check_gradient(want, dy.cpu(), t.cpu(), V, 1.5, dtype, what=T)
    same(fp8q.embedding_backward(far(dy, ld), t, V, 1.5, dtype=dtype), want, "dy far apart")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", SORTED)
def test_far_rows_of_the_table(T, dtype):
    """Rows 2^31 elements apart: filled with zeros (row 1), stored by the sums and by the join, and added to."""
    V, C = 4, 96
    print("far table", T, dtype, flush=True)
    g = torch.Generator().manual_seed(T)
    # (row 3 has one chunk's run at the end of the order, rows 0 and 2 run over many)
    t = torch.randint(0, 2, (T,), generator=g) * 2
    t[5::T // 3] = 3
    t = t.to(DEV)
    dy = rand(T, C, seed=T + 3)
    want = fp8q.embedding_backward(dy, t, V, 1.5, dtype=dtype)
    check_gradient(want, dy.cpu(), t.cpu(), V, 1.5, dtype, what=T)
    there = far(torch.ones_like(want), FAR)
    fp8q.embedding_backward(dy, t, V, 1.5, dtype=dtype, dweight=there)
    same(there.contiguous(), want, "a far table's gradient")
    assert not bool(there[1].any())
    twice = want.clone()
    for into in (twice, there):
        fp8q.embedding_backward(dy, t, V, 1.5, dtype=dtype, dweight=into, accumulate=True)
    same(there.contiguous(), twice, "added to")


@pytest.mark.parametrize("T", [700, 17500])
def test_large_gradient(T):
    """A table of just under 2^33 elements, in bf16: rows at its end are summed, filled and left."""
    V, C = (1 << 22) - 1, 2048
    print("large gradient", T, flush=True)
    n = T // 5
    dy, tokens = rand(T, C), torch.tensor([V - 1, V - 2, 7, V - 1, V] * n, device=DEV)
    dw = torch.ones((V, C), dtype=BF16, device=DEV)
    fp8q.embedding_backward(dy, tokens, V, dtype=BF16, dweight=dw)
    d = dy.double().view(n, 5, C)
    for row, terms in ((V - 1, (d[:, 0], d[:, 3])), (V - 2, (d[:, 1],)), (7, (d[:, 2],))):
        # fp32 sums of m = len(terms) n rows, each addition off by half a unit of a partial sum ((1 + 2^-24)^m - 1 is at
        # most m 2^-24 (1 + 2^-11) here), then one rounding to bf16, of the error, too
        exact, most = sum(x.sum(0) for x in terms), sum(x.abs().sum(0) for x in terms)
        bound = 2.0 ** -8 * exact.abs() + (1 + 2.0 ** -7) * len(terms) * n * 2.0 ** -24 * most
        assert bool(((dw[row].double() - exact).abs() <= bound).all()), row
    for rows in (slice(0, 7), slice(8, 1 << 21), slice(1 << 21, V - 2)):
        assert not bool(dw[rows].any())


def test_workspaces_on_two_streams():
    """Other inputs on each of two streams at once, of sizes whose calls take a workspace: the small and the large
    sort with runs over many chunks, and split rows of logits."""
    def inputs(seed):
        g = torch.Generator().manual_seed(seed)
        made = []
        for T, V, C, accumulate in ((600, 90, 320, False), (9001, 700, 128, True), (17000, 2000, 64, False)):
            made.append((rand(T, C, seed=seed + T), tokens_of(T, V, seed + T).to(DEV), V, rand(V, C, F32, seed=seed), accumulate))
        x = torch.randn(4, 90000, generator=g).bfloat16().to(DEV)
        return made, x, torch.randint(0, 90000, (4,), generator=g).to(DEV)

    def run(state):
        made, x, tokens = state
        out = [fp8q.embedding_backward(dy, t, V, 0.5, dweight=old.clone(), accumulate=a) for dy, t, V, old, a in made]
        return out + list(fp8q.top_logprobs(x, tokens, 9))

    assert fp8q.lib().fp8q_top_logprobs_workspace(4, 90000, 9) > 0
    states = [inputs(41), inputs(42)]
    want = [run(s) for s in states]
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((i, run(states[i])))
    torch.cuda.synchronize()
    for i, results in got:
        for j, (a, b) in enumerate(zip(results, want[i])):
            same(a, b, "stream %d, output %d" % (i, j))
    assert not torch.equal(want[0][0], want[1][0])
