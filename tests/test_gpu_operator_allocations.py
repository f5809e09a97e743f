"""The operators' results and workspaces are allocated as torch allocates: what listens to torch's dispatcher sees them,
and memory that torch is asked to fill is filled."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from launched import kernels
    from torch.utils._python_dispatch import TorchDispatchMode

    from paper_1811_12843_gb300 import operators as ops

    class Seen(TorchDispatchMode):
        """How many tensors on the GPU are allocated."""
        count = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            r = func(*args, **(kwargs or {}))
            if func in (torch.ops.aten.empty.memory_format, torch.ops.aten.empty_strided.default):
                self.count += r.is_cuda
            return r

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def calls():
    """(name, call, tensors that it allocates) for [rows, columns] and for [groups, rows, columns]."""
    gen = torch.Generator("cuda").manual_seed(3)

    def randn(*shape, dtype=BF16):
        return torch.randn(shape, device="cuda", generator=gen).to(dtype)

    for lead in ((), (3,)):
        x, w, g = randn(*lead, 130, 264), randn(*lead, 72, 264), 1 + 0.1 * randn(*lead, 264, dtype=F32)
        dy = randn(*lead, 130, 72)
        mean, rstd = x.float().mean(-1), x.float().var(-1).rsqrt()
        xc, pc = ops.checkpoint_rows(x), ops.checkpoint_rows(dy)
        yield "rmsnorm", lambda: ops.rmsnorm(x, g, residual=x, e4m3=True, keep=True), 4
        yield "rmsnorm_backward", lambda: ops.rmsnorm_backward(x, x, rstd, g), 2
        yield "quantize_rows", lambda: ops.quantize_rows(x), 2
        yield "linear", lambda: ops.linear(x, w, keep=True), 2
        yield "linear_backward", lambda: ops.linear_backward(dy, x, w, act="gelu", pre=dy), 4  # (and its workspace)
        yield "layernorm", lambda: ops.layernorm(x, g, g, residual=x, e4m3=True, keep="int8"), 7
        yield "layernorm_backward", lambda: ops.layernorm_backward(x, xc, mean, rstd, g), 3
        yield "checkpoint_rows", lambda: ops.checkpoint_rows(x), 2
        yield "restore_rows", lambda: ops.restore_rows(xc), 1
        yield "linear keeping", lambda: ops.linear(x, w, keep="int8"), 3
        yield "backward over checkpoints", lambda: ops.linear_backward(dy, xc, w, act="gelu", pre=pc), 4


def tensors(v):
    if torch.is_tensor(v):
        return [v]
    return [t for u in v if u is not None for t in tensors(u)]


def same(a, b):
    a, b = tensors(a), tensors(b)
    return len(a) == len(b) and all(p.dtype is q.dtype and p.shape == q.shape and p.stride() == q.stride() and
                                    torch.equal(p.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8))
                                    for p, q in zip(a, b))


def test_a_dispatch_mode_sees_every_tensor():
    for name, call, count in calls():
        ref = call()
        with Seen() as seen:
            got = call()
        assert seen.count >= count, (name, seen.count)
        assert same(got, ref), name


def test_the_profiler_sees_every_tensor():
    for name, call, count in calls():
        with torch.autograd.profiler.profile() as p:
            call()
        events = [e for e in p.function_events if e.name in ("aten::empty", "aten::empty_strided")]
        assert len(events) >= count, (name, len(events))


def test_memory_is_filled_where_torch_is_asked_to():
    """A kernel more for each tensor, before the call's own: torch fills it, the call writes it."""
    before = torch.are_deterministic_algorithms_enabled(), torch.utils.deterministic.fill_uninitialized_memory
    for name, call, count in calls():
        ref, plain = call(), kernels(call)
        try:
            torch.use_deterministic_algorithms(True)
            torch.utils.deterministic.fill_uninitialized_memory = True
            filled, got = kernels(call), call()
            torch.utils.deterministic.fill_uninitialized_memory = False
            unfilled = kernels(call)
        finally:
            torch.use_deterministic_algorithms(before[0])
            torch.utils.deterministic.fill_uninitialized_memory = before[1]
        assert len(filled) >= len(plain) + count and len(unfilled) == len(plain), (name, len(plain), len(filled))
        assert same(got, ref), name


def test_inference_mode_and_no_grad_give_the_same():
    for name, call, _ in calls():
        ref = call()
        with torch.inference_mode():
            got = call()
            assert same(got, ref) and all(t.is_inference() for t in tensors(got) if t.data_ptr()), name
        with torch.no_grad():
            assert same(call(), ref), name
