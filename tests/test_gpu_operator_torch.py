"""The operators beside torch's own bookkeeping: writes are seen by autograd and by copy-on-write, and no
gradient is lost without a word."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_1811_12843_gb300 as L
    from paper_1811_12843_gb300 import operators as ops

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def randn(*shape, dtype=BF16):
    return torch.randn(*shape, device="cuda").to(dtype)


def in_place(t):
    """The calls that write into a tensor of the caller's, [24, 64]."""
    x, w, g = randn(24, 64), randn(64, 64), torch.ones(64, device="cuda")
    return [lambda: ops.rmsnorm(x, g, residual=t, sum_out=t), lambda: ops.linear(x, w, residual=t, out=t),
            lambda: ops.linear(x, w, out=t)]


def test_a_write_moves_the_version():
    t = randn(24, 64)
    for call in in_place(t):
        before = t._version
        call()
        assert t._version == before + 1
    inputs = [randn(24, 64), randn(64, 64)]
    ops.linear(*inputs)
    assert [i._version for i in inputs] == [0, 0]


def test_a_graph_that_saved_the_tensor_refuses_its_new_values():
    for i in range(3):
        leaf = randn(24, 64).requires_grad_(True)
        s = leaf * 2
        z = (s * s).sum()
        with torch.no_grad():
            in_place(s)[i]()
        with pytest.raises(RuntimeError, match="inplace"):
            z.backward()


def test_a_lazy_clone_is_a_tensor_of_its_own():
    for i in range(3):
        t = randn(24, 64)
        before, clone = t.clone(), torch._lazy_clone(t)
        in_place(clone)[i]()
        torch.cuda.synchronize()
        assert torch.equal(t, before) and not torch.equal(clone, before)


def test_inference_tensors_are_written_in_inference_mode_alone():
    with torch.inference_mode():
        t = randn(24, 64)
        for call in in_place(t):
            call()
    before = t.clone()
    for call in in_place(t):
        with pytest.raises(L.LipzError, match="inference"):
            call()
    assert torch.equal(t, before)


def test_a_gradient_is_refused_where_it_would_be_lost():
    x, w, g = randn(24, 64), randn(32, 64), torch.ones(64, device="cuda")
    bias, rstd, q = torch.zeros(32, device="cuda"), torch.ones(24, device="cuda"), ops.quantize_rows

    def grad(t):
        return t.detach().clone().requires_grad_(True)

    calls = [lambda f: ops.rmsnorm(f(x), g), lambda f: ops.rmsnorm(x, f(g)),
             lambda f: ops.rmsnorm(x, g, residual=f(x)), lambda f: q(f(x)), lambda f: ops.linear(f(x), w),
             lambda f: ops.linear(x, f(w)), lambda f: ops.linear(x, w, f(bias)),
             lambda f: ops.linear(x, w, residual=f(randn(24, 32))),
             lambda f: ops.rmsnorm_backward(f(x), x, rstd, g), lambda f: ops.linear_backward(randn(24, 32), x, f(w))]
    for call in calls:
        call(lambda t: t)
        with pytest.raises(L.LipzError, match="gradient") as e:
            call(grad)
        assert e.value.code == L.LIPZ_ERR_INVALID
        with torch.no_grad():
            call(grad)
        with torch.inference_mode():
            call(grad)
        call(lambda t: grad(t).detach())
