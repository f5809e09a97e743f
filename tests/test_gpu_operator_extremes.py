"""The residual-block operators at the ends of their types' ranges: finite inputs whose results are finite by
the formulas give them."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_1811_12843_gb300 import operators as ops
    from test_gpu_operators import within

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


@pytest.mark.parametrize("act", ["tanh", "gelu", "silu"])
@pytest.mark.parametrize("n", [256, 250])
def test_slopes_at_huge_pre_activations(act, n):
    """The slopes' limits are 0 and 1 (tanh: 0), and reached long before the type ends."""
    big = [1e4, 1e10, 1e15, 4e18, 2e19, 1e20, 1e30, 3e38]
    pre = torch.tensor(big + [-b for b in big], device="cuda").repeat(n // 16 + 1)[:n].repeat(40, 1).to(BF16)
    dy = torch.ones(40, n, device="cuda", dtype=BF16)
    w = torch.eye(n, device="cuda", dtype=BF16)
    dx, _, db = ops.linear_backward(dy, dy, w, act=act, pre=pre)
    slope = torch.zeros_like(pre) if act == "tanh" else (pre > 0).to(BF16)
    assert torch.equal(dx, slope)
    assert torch.equal(db, slope.float().sum(dim=0))


@pytest.mark.parametrize("rows", [1, 3, 20, 300])
@pytest.mark.parametrize("scale", [2e19, 1e-22])
def test_scales_multiply_one_after_the_other(rows, scale):
    """Scales whose product leaves fp32's normal range, beside sums that bring the result back into it or are
    zero: the same in the kernels for few, some and many rows."""
    k, n = 256, 96
    x, w = torch.ones(rows, k, device="cuda"), torch.zeros(n, k, device="cuda")
    if scale > 1:
        w[::2, 7] = 0.25
    else:
        w[::2] = torch.arange(k, device="cuda").remainder(15) + 1.0
    xs, ws = torch.full((rows,), scale, device="cuda"), torch.full((n,), scale, device="cuda")
    y, _ = ops.linear(x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn), x_scale=xs, w_scale=ws, out_dtype=F32)
    ref = (x.to(F64) @ w.to(F64).T) * xs.to(F64)[:, None] * ws.to(F64)
    assert ref.abs().max() < 3e38 and (ref[:, ::2] > 0).all()
    within(y, ref, 2.0 ** -20 * ref.abs() + 2.0 ** -148)


@pytest.mark.parametrize("rows,dim", [(5, 64), (700, 256), (700, 2056), (700, 1001), (4, 16383)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_backward_of_tiny_rows(rows, dim, dtype):
    """rstd of 1e22: its square is infinite, the gradient is not."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    s = (torch.randn((rows, dim), generator=gen, device="cuda") * 1e-22).to(dtype)
    dy = (torch.randn((rows, dim), generator=gen, device="cuda") * 1e-3).to(dtype)
    w = 1 + 0.1 * torch.randn(dim, generator=gen, device="cuda")
    rstd = s.to(F64).square().mean(dim=1).rsqrt().float()
    dx, dw = ops.rmsnorm_backward(dy, s, rstd, w)
    g, r, s64 = dy.to(F64) * w.to(F64), rstd.to(F64)[:, None], s.to(F64)
    ref = r * (g - (s64 * r) * (r * (g * s64).mean(dim=1, keepdim=True)))
    size = r * (g.abs() + (s64 * r).abs() * (r * (g * s64).abs().mean(dim=1, keepdim=True)))
    rounding = 2.0 ** -8 if dtype == BF16 else 2.0 ** -23
    within(dx, ref, rounding * ref.abs() + ((dim + 16) * 2.0 ** -24 + 2.0 ** -20) * size, "dx")
    within(dw, (dy.to(F64) * s64 * r).sum(dim=0),
           (rows + 16) * 2.0 ** -23 * (dy.to(F64) * s64 * r).abs().sum(dim=0), "dweight")
