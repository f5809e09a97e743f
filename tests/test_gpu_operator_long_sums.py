"""Products over very many k, with results in bf16: the tensor cores' additions truncate, and what that loses of
a sum whose terms have one sign grows with k. Every result must be the rounding of a value within 2^-13 of the sum: off
by no more than half of bf16's unit where it lies, and that."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_1811_12843_gb300 import operators as ops

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def positive(seed, *shape):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(shape, generator=gen, device="cuda").add_(0.25).to(BF16)


def product64(a, b, at=65536):
    """a [m, k] b [n, k]^T in 64 bits."""
    return sum(a[:, i:i + at].to(F64) @ b[:, i:i + at].to(F64).T for i in range(0, a.shape[1], at))


def near(got, ref):
    unit = torch.exp2(torch.frexp(got.to(F64)).exponent.to(F64) - 8)
    off = (got.to(F64) - ref).abs() - unit / 2
    assert (off <= 2.0 ** -13 * ref).all(), (off / ref).max().item()


@pytest.mark.parametrize("rows,n,k", [(128, 64, 1 << 20), (40, 200, 1 << 20), (300, 320, 500000), (2048, 2048, 200000)])
def test_linear(rows, n, k):
    x, w = positive(1, rows, k), positive(2, n, k)
    residual = torch.zeros(rows, n, device="cuda", dtype=BF16)
    y, pre = ops.linear(x, w, residual=residual, keep=True)
    m = min(rows, 128)
    ref = product64(x[:m], w[-64:])
    near(y[:m, -64:], ref)
    assert torch.equal(y, pre)


@pytest.mark.parametrize("rows,n,k", [(260, 192, 1 << 20), (2048, 2048, 400000)])
def test_linear_8_bits(rows, n, k):
    x, w = positive(3, rows, k).to(torch.float8_e4m3fn), positive(4, n, k).to(torch.float8_e4m3fn)
    one = torch.ones(2048, device="cuda")
    y, _ = ops.linear(x, w, x_scale=one[:rows], w_scale=one[:n])
    near(y[:64, :64], product64(x[:64], w[:64]))


@pytest.mark.parametrize("rows,n,k", [(2048, 2048, 17000), (2050, 1999, 17000), (6000, 200, 20001)])
@pytest.mark.parametrize("act,apart", [("none", 0), ("silu", 3)])
def test_residuals_beside_long_sums(rows, n, k, act, apart):
    """Terms of both signs, with every part of the epilogue: within 2^-8 of the result, 2^-18 of the activation and
    (k / 16 + 16) 2^-22 of the sum of magnitudes, as shorter sums are."""
    gen = torch.Generator(device="cuda").manual_seed(8)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(BF16)

    x, w, bias = randn(rows, k), randn(n, k) * k ** -0.5, randn(n).float()
    stream = randn(rows, n + apart)[:, :n]
    before = stream.clone()
    y, pre = ops.linear(x, w, bias, act=act, residual=stream, out=stream, keep=True)
    assert y is stream
    a, b = x[-150:].to(F64), w[-90:].to(F64)
    u, mag = a @ b.T + bias[-90:].to(F64), a.abs() @ b.abs().T + bias[-90:].abs().to(F64)
    err = (k / 16 + 16) * 2.0 ** -22 * mag
    f = u if act == "none" else u * torch.sigmoid(u)
    out = f + before[-150:, -90:].to(F64)
    assert ((y[-150:, -90:].to(F64) - out).abs() <= 2.0 ** -8 * out.abs() + 1.2 * err + 2.0 ** -18 * f.abs()).all()
    assert ((pre[-150:, -90:].to(F64) - u).abs() <= 2.0 ** -8 * u.abs() + err).all()


@pytest.mark.parametrize("rows,n,k", [(300000, 2048, 2048), (200001, 1024, 520)])
def test_weight_gradient(rows, n, k):
    dy, x, w = positive(5, rows, n), positive(6, rows, k), positive(7, n, k)
    dx, dw, db = ops.linear_backward(dy, x, w)
    near(dw[-64:, :64], product64(dy[:, -64:].T, x[:, :64].T))
    near(dx[-64:, :64], product64(dy[-64:], w[:, :64].T))
    only = ops.linear_backward(dy, x, w, want_dx=False, want_db=False)[1]
    assert torch.equal(only, dw)
    only = ops.linear_backward(dy, x, w, want_dw=False)
    assert torch.equal(only[0], dx) and torch.equal(only[2], db)
