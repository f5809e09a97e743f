"""The activations and their slopes in fp32, from pre-activations that are exact in it, over the whole range where
they are not 0, 1 or u. Errors to expect: the exponential, reciprocal and product 2^-22, 2^-23 and 2^-24 of the
value; and the exponent's rounding, 2^-24 for each of its operations times the exponent, |u| for silu and tanh and
|v| = |u (GELU_1 + GELU_3 u^2)| for gelu, whose own three roundings come on top. Slopes: the same of the sizes of
their terms, and 2^-23 where 1 - g is taken from a g near 1."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_1811_12843_gb300 import operators as ops

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
G1 = 2 * math.sqrt(2 / math.pi)
G3 = G1 * 0.044715


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def points():
    """Every bf16 value whose results are neither constant nor u itself, of both signs."""
    u = torch.arange(0x3000, 0x42A1, device="cuda", dtype=torch.int16).view(BF16)  # 4.7e-10 to 80
    return torch.cat([u, -u])


def sigmoid64(v):
    e = torch.exp(-v.abs())
    return torch.where(v >= 0, torch.ones_like(e), e) / (1 + e)


def reference(act, u):
    """(value, its error, slope, its error)"""
    if act == "tanh":
        t, e = torch.tanh(u), torch.exp(-2 * u.abs())
        slope = 4 * e / (1 + e) ** 2
        return t, 2.0 ** -20 * t.abs(), slope, slope * (2.0 ** -20 + 2 * u.abs() * 2.0 ** -22)
    c1, c3 = (G1, G3) if act == "gelu" else (1.0, 0.0)
    v, ds = u * (c1 + c3 * u * u), c1 + 3 * c3 * u * u
    g = sigmoid64(v)
    rel = 2.0 ** -21 + v.abs() * 2.0 ** (-23 if act == "silu" else -21)
    near = 1 - g
    slope = g + u * g * near * ds
    size = g * (1 + u.abs() * near * ds)
    return u * g, rel * (u * g).abs(), slope, 2 * rel * size + g * u.abs() * ds * 2.0 ** -22


@pytest.mark.parametrize("act", ["tanh", "gelu", "silu"])
@pytest.mark.parametrize("rows", [1, 20, 700])
def test_values(act, rows):
    u = points()
    w = torch.zeros(u.numel(), 32, device="cuda", dtype=BF16)
    w[:, 3] = u
    x = torch.ones(rows, 32, device="cuda", dtype=BF16)
    y, _ = ops.linear(x, w, act=act, out_dtype=F32)
    value, error, _, _ = reference(act, u.to(F64))
    off = (y.to(F64) - value).abs() - error
    assert (off <= u.to(F64).abs() * 2.0 ** -126).all(), (u[off.argmax() % u.numel()].item(), off.max().item())


@pytest.mark.parametrize("act", ["tanh", "gelu", "silu"])
def test_slopes(act):
    u = points()
    one = torch.ones(1, u.numel(), device="cuda", dtype=BF16)
    _, _, db = ops.linear_backward(one, one[:, :8], torch.zeros(u.numel(), 8, device="cuda", dtype=BF16), act=act,
                                   pre=u[None], want_dx=False, want_dw=False)
    _, _, slope, error = reference(act, u.to(F64))
    off = (db.to(F64) - slope).abs() - error
    assert (off <= u.to(F64).abs() * 2.0 ** -120).all(), (u[off.argmax()].item(), off.max().item())
