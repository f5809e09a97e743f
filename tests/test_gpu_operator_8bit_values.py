"""The 8-bit values of quantize_rows and rmsnorm: q = e4m3(x / scale), to nearest even, for rows of every
magnitude that their types hold.

The quotient is taken in 64 bits from the scale that the call returned. A value whose quotient is exactly
halfway between two e4m3 values must go to the even one; one that is nearer to halfway than the quotient's
own rounding to fp32 (2^-24 of at most 16 steps) may go to either."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_1811_12843_gb300 import operators as ops

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64

# a few rows, many short ones, many longer ones, widths off the 16-byte grid by units and by elements, and
# rows that are read twice
SHAPES = [(9, 64), (9, 784), (9, 1001), (700, 64), (700, 784), (700, 2056), (700, 1001), (620, 16378), (12, 20000),
          (12, 20001)]


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def check_values(q, scale, x):
    q, x, scale = q.to(F64), x.to(F64), scale.to(F64)
    ref = (x.abs().amax(dim=-1) / 448).clamp(min=2.0 ** -126)
    assert ((scale - ref).abs() <= 2.0 ** -23 * ref).all()
    v = x / scale[..., None]
    step = torch.exp2((torch.frexp(v).exponent - 1).clamp(min=-6).to(F64) - 3)
    n = v / step
    off = (n - n.floor() - 0.5).abs()
    open_ = (off > 0) & (off <= 2.0 ** -20)
    bad = (q != torch.round(n) * step) & ~open_
    assert not bad.any(), (int(bad.sum()), q[bad][:4], v[bad][:4])


def extreme_rows(rows, dim, dtype):
    """Rows of random values at magnitudes from the type's largest to its smallest, in turn."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = torch.rand((rows, dim), generator=gen, device="cuda", dtype=F64) * 2 - 1
    top = [float(torch.finfo(dtype).max), 2.0 ** 127, 1.7 * 2.0 ** 126, 2.0 ** 126, 0.9 * 2.0 ** 126, 1e30, 1.0, 3e-6,
           1e-30, 448 * 2.0 ** -126, 1e-37, 1e-40]
    x = x * torch.tensor(top, dtype=F64, device="cuda").repeat(rows // len(top) + 1)[:rows, None]
    x[:, 0] = x[:, 0].sign() * torch.tensor(top, dtype=F64, device="cuda").repeat(rows // len(top) + 1)[:rows]
    return x.to(dtype).nan_to_num()


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_any_magnitude_keep_their_values(rows, dim, dtype):
    x = extreme_rows(rows, dim, dtype)
    q, scale = ops.quantize_rows(x)
    check_values(q, scale, x)
    assert (q.float()[:, 0].abs() == 448).sum() >= rows * 2 // 3  # (all but the subnormal rows')


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("odd", [1, 3])
def test_ties_go_to_the_even_value(rows, dim, dtype, odd):
    """Scales odd 2^j, and values halfway between two of e4m3's among the others."""
    halfway = torch.tensor([17.0, 19, 21, 23, 25, 27, 29, 31, 34, 38, 42, 1.0625, 0.5 * 2.0 ** -9, 1.5 * 2.0 ** -9,
                            424, -17, -25, 5, 448], dtype=F64, device="cuda")
    v = halfway.repeat(dim // len(halfway) + 1)[:dim].repeat(rows, 1)
    v[:, 0] = 448
    j = torch.arange(rows, device="cuda").remainder(200).sub(100).to(F64)
    x = v * odd * torch.exp2(j)[:, None]
    exact = x.to(dtype)
    assert torch.equal(exact.to(F64), x)
    q, scale = ops.quantize_rows(exact)
    assert torch.equal(scale.to(F64), odd * torch.exp2(j))
    check_values(q, scale, exact)


@pytest.mark.parametrize("rows,dim", SHAPES)
def test_ties_beside_any_scale(rows, dim):
    """Every row's scale is another odd number: the quotients of ties are exact, the scales' reciprocals not."""
    halfway = torch.tensor([17.0, 19, 21, 23, 25, 27, 29, 31, 34, 38, 42, 1.0625, 424, 5.25, -17, 448], dtype=F64,
                           device="cuda")
    v = halfway.repeat(dim // len(halfway) + 1)[:dim].repeat(rows, 1)
    v[:, 0] = 448
    odd = torch.arange(rows, device="cuda").mul(2).add(101).to(F64)
    x = (v * odd[:, None]).to(F32)
    q, scale = ops.quantize_rows(x)
    assert torch.equal(scale.to(F64), odd)
    check_values(q, scale, x)


@pytest.mark.parametrize("rows,dim", [s for s in SHAPES if s[1] <= 16384])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top", [448.0, 448 * 3 * 2.0 ** -20, 448 * 2.0 ** 119])
def test_the_norm_in_8_bits(rows, dim, dtype, top):
    """Rows of +-1 have the reciprocal root 1, so that the norm's results are the weights."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    sign = torch.randint(0, 2, (rows, dim), generator=gen, device="cuda").mul(2).sub(1)
    w = torch.rand(dim, generator=gen, device="cuda").mul(2).sub(1).mul(top)
    ties = torch.tensor([17.0, 19, 25, 31, 1.0625, 424], device="cuda") * (top / 448)
    w[1:1 + len(ties)] = ties
    w[0] = top
    r = ops.rmsnorm(sign.to(dtype), w, eps=0.0, e4m3=True, keep=True)
    assert (r.rstd == 1).all()
    check_values(r.y, r.scale, sign.to(F64) * w.to(F64))
