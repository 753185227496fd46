"""The tensors that calls make are those that torch.empty makes: seen by dispatch
modes and the profiler, filled where torch fills new memory, of the current
inference mode, and from the caller's stream."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import paper_2609_22870_amd as fp8q

from _ops import DEV, same

pytestmark = pytest.mark.gpu

B1 = fp8q.BLOCK_1x128


class Seen(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.names = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.names.append(func.name())
        return func(*args, **(kwargs or {}))


def inputs():
    g = torch.Generator().manual_seed(71)
    x = torch.randn(64, 256, generator=g).bfloat16().to(DEV)
    w = torch.ones(256, dtype=torch.bfloat16, device=DEV)
    return x, w


# (call, new tensors)
CALLS = {
    "quantize": (lambda x, w: fp8q.quantize(x, B1), 2),
    "rmsnorm": (lambda x, w: fp8q.rmsnorm(x, w, 1e-6), 2),
    "rmsnorm_quantize": (lambda x, w: fp8q.rmsnorm_quantize(x, w, 1e-6, residual=x), 4),
    "gated_backward": (lambda x, w: fp8q.gated_backward(x[:, :128], x), 4),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_dispatch_modes_see_the_new_tensors(name):
    call, new = CALLS[name]
    x, w = inputs()
    want = call(x, w)
    with Seen() as seen:
        got = call(x, w)
    assert sum(n.startswith("aten::empty.") for n in seen.names) == new, seen.names
    for a, b in zip(got, want):
        same(a, b, name)


@pytest.mark.parametrize("name", list(CALLS))
def test_the_profiler_sees_the_new_tensors(name):
    call, new = CALLS[name]
    x, w = inputs()
    call(x, w)
    torch.cuda.synchronize()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as p:
        call(x, w)
    assert sum(e.name == "aten::empty" for e in p.events()) == new


@pytest.fixture
def deterministic():
    before = torch.are_deterministic_algorithms_enabled(), torch.utils.deterministic.fill_uninitialized_memory
    yield
    torch.use_deterministic_algorithms(before[0])
    torch.utils.deterministic.fill_uninitialized_memory = before[1]


@pytest.mark.parametrize("fill", [False, True])
def test_deterministic_fill(fill, deterministic):
    """The loss's workspace holds places for the parts of split rows.  200 rows are not
    split, so those keep what the allocation holds: with torch's fill, 255 in every
    byte, also where the memory held something else before."""
    T, V = 200, 256
    g = torch.Generator().manual_seed(72)
    args = [torch.randn(T, V, generator=g).to(DEV), torch.randint(0, V, (T,), generator=g).to(DEV)]
    args += [torch.zeros(T, device=DEV), torch.ones(T, device=DEV), torch.ones(T, device=DEV)]
    need = fp8q.lib().fp8q_policy_loss_workspace(T, V)
    fp8q.policy_loss(*args, 0.8, 1.2)
    torch.cuda.synchronize()
    old = torch.full((need,), 7, dtype=torch.uint8, device=DEV)
    where = old.data_ptr()
    del old  # the allocator's next block of this size
    torch.use_deterministic_algorithms(fill)
    torch.utils.deterministic.fill_uninitialized_memory = fill
    fp8q.policy_loss(*args, 0.8, 1.2)
    torch.use_deterministic_algorithms(False)
    now = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert now.data_ptr() == where
    rest = now[(4 * T + 15) // 16 * 16:].cpu()
    assert bool((rest == (255 if fill else 7)).all())


def test_inference_mode_and_stream():
    x, w = inputs()
    want = fp8q.rmsnorm_quantize(x, w, 1e-6, residual=x)
    assert not any(t.is_inference() or t.requires_grad for t in want)
    torch.cuda.synchronize()
    with torch.inference_mode(), torch.cuda.stream(torch.cuda.Stream()):
        got = fp8q.rmsnorm_quantize(x, w, 1e-6, residual=x)
        plain = torch.empty(4, device=DEV)
    torch.cuda.synchronize()
    assert all(t.is_inference() == plain.is_inference() for t in got)
    for a, b in zip(got, want):
        assert a.is_contiguous() and a.device == b.device and a.dtype == b.dtype
        same(a, b, "inference mode")
