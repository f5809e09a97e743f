"""The residual-block operators against their definitions in 64 bits.

Tolerances are element by element, from the number formats: a result rounded once to bf16 is within
2^-8 of its size (2^-24 in fp32), e4m3 within 2^-4 of it or half of its smallest step, and a sum of
products over k within (k / 16 + 16) 2^-22 of the sum of their magnitudes (the tensor cores add 16
products at a time and truncate to fp32; chains of fp32 additions stay below that too). The activations'
hardware approximations are good to 2^-18. Where a delta is rounded to bf16 before a product, the sum
of magnitudes times 2^-8 comes on top.
"""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_1811_12843_gb300 as L
    from paper_1811_12843_gb300 import operators as ops

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3 = torch.float8_e4m3fn
ACTS = ["none", "relu", "lrelu", "tanh", "gelu", "silu"]
ROUND = {BF16: 2.0 ** -8, F32: 2.0 ** -23}
SLOPE = 0.3


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def randn(seed, shape, std=1.0, dtype=BF16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def d(t):
    return t.to(F64)


def within(got, ref, tol, what=""):
    """Every element within tol of ref; NaN exactly where ref has it."""
    got = d(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.equal(got.isnan(), ref.isnan()), what
    bad = ((got - ref).abs() > tol) & ~ref.isnan() & (got != ref)
    if bad.any():
        i = int(((got - ref).abs() / tol).nan_to_num(0.0).argmax())
        raise AssertionError("%s: %d of %d elements off, worst %r for %r (tolerance %r) at %d" % (
            what, int(bad.sum()), bad.numel(), got.flatten()[i].item(), ref.flatten()[i].item(),
            tol.expand_as(ref).flatten()[i].item(), i))


def act64(act, u):
    if act == "relu":
        return torch.where(u < 0, torch.zeros_like(u), u)
    if act == "lrelu":
        return torch.where(u > 0, u, SLOPE * u)
    if act == "tanh":
        return torch.tanh(u)
    if act == "gelu":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    if act == "silu":
        return u * torch.sigmoid(u)
    return u


def slope64(act, u):
    if act in ("relu", "lrelu"):
        return torch.where(u > 0, 1.0, 0.0 if act == "relu" else SLOPE).to(F64)
    v = u.detach().clone().requires_grad_(True)
    act64(act, v).sum().backward()
    return v.grad if v.grad is not None else torch.ones_like(u)


def sum_error(k):
    return (k / 16 + 16) * 2.0 ** -22


# ---- rmsnorm ------------------------------------------------------------------------------------
# one element, widths around a warp's vectors and a block's, ragged widths, the widest
NORM_SHAPES = [(1, 1, 1), (1, 1, 4096), (1, 3, 7), (1, 5, 64), (1, 37, 256), (3, 11, 257), (1, 9, 784),
               (2, 400, 1000), (1, 700, 2056), (1, 6, 4104), (1, 320, 8192), (2, 3, 8191), (1, 330, 16384),
               (1, 4, 16383), (144, 100, 256), (1, 1, 16384), (1, 0, 64), (0, 4, 64)]


def norm_shape(groups, *dims):
    return dims if groups == 1 else (groups,) + dims


def norm_ref(x, residual, weight, eps):
    s = d(x) if residual is None else d(x) + d(residual)
    rstd = (s.square().mean(dim=-1) + eps).rsqrt()
    return s, rstd, s * rstd[..., None] * d(weight)[..., None, :]


def check_norm(r, x, residual, weight, eps, e4m3, keep):
    s, rstd, y = norm_ref(x, residual, weight, eps)
    dim = x.shape[-1]
    rel = (dim + 16) * 2.0 ** -24 + 2.0 ** -21  # a sum of squares, its root, two products
    if e4m3:
        scale = (y.abs().amax(dim=-1) / 448).clamp(min=2.0 ** -126)
        within(r.scale, scale, rel * scale, "scale")
        v = y / scale[..., None]
        within(r.y, v, 2.0 ** -4 * v.abs() * (1 + 2 * rel) + 2.0 ** -10 + 448 * rel, "y")
    else:
        assert r.scale is None
        within(r.y, y, (ROUND[x.dtype] + rel) * y.abs() + 1e-37, "y")
    if residual is None:
        assert r.sum is x
    else:
        within(r.sum, s, ROUND[x.dtype] * s.abs(), "sum")
    if keep:
        within(r.rstd, rstd, rel * rstd, "rstd")
    else:
        assert r.rstd is None


@pytest.mark.parametrize("groups,rows,dim", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,e4m3,keep", [(False, False, True), (True, True, False),
                                                (True, False, True)])
def test_rmsnorm(groups, rows, dim, dtype, residual, e4m3, keep):
    x = randn(1, norm_shape(groups, rows, dim), 2.0, dtype)
    res = randn(2, norm_shape(groups, rows, dim), 3.0, dtype) if residual else None
    w = 1 + randn(3, norm_shape(groups, dim), 0.2, F32)
    if rows == 0 or groups == 0:
        r = ops.rmsnorm(x, w, residual=res, e4m3=e4m3, keep=keep)
        assert r.y.shape == x.shape
        return
    r = ops.rmsnorm(x, w, residual=res, eps=1e-5, e4m3=e4m3, keep=keep)
    check_norm(r, x, res, w, 1e-5, e4m3, keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [256, 250, 6000])
def test_rmsnorm_strides_and_places(dtype, dim):
    """Rows cut from wider ones off the 16-byte grid, groups woven row by row, a shared residual and
    weight, the residual stream updated in place."""
    rows, groups = 33, 4
    wide = randn(4, (rows, groups, dim + 5), 1.0, dtype)
    x = wide[:, :, 3:3 + dim].permute(1, 0, 2)
    res = randn(5, (1, rows, dim), 1.0, dtype).expand(groups, rows, dim)
    w = (1 + randn(6, (1, dim), 0.1, F32)).expand(groups, dim)
    r = ops.rmsnorm(x, w, residual=res, e4m3=True, keep=True)
    check_norm(r, x, res, w, 1e-6, True, True)
    own, before = randn(7, (groups, rows, dim), 1.0, dtype), None
    before = own.clone()
    r = ops.rmsnorm(x, w, residual=own, sum_out=own)
    assert r.sum is own
    check_norm(r, x, before, w, 1e-6, False, False)


def test_rmsnorm_extreme_rows():
    """Zero rows, subnormal and huge rows, NaN and infinity: each stays in its row."""
    x = randn(8, (8, 512), 1.0, F32)
    x[1] = 0
    x[2] *= 1e-41
    x[3] *= 1e15
    x[4, 7] = float("nan")
    x[5, 500] = float("inf")
    w = 1 + randn(9, (512,), 0.1, F32)
    for dtype in (F32, BF16):
        xs = x.to(dtype)
        r = ops.rmsnorm(xs, w, e4m3=False)
        q = ops.rmsnorm(xs, w, e4m3=True)
        ok = [0, 1, 2, 3, 6, 7]
        assert torch.isfinite(r.y[ok]).all() and torch.isfinite(q.y.float()[ok]).all()
        assert (r.y[1] == 0).all() and (q.y.float()[1] == 0).all() and q.scale[1] == 2.0 ** -126
        assert r.y[4].isnan().all() and q.y.float()[4].isnan().all() and q.scale[4].isnan()
        assert r.y[5, 500].isnan() and (r.y[5, :500] == 0).all()
        assert q.scale[5].isnan() and q.y.float()[5].isnan().all()
        _, _, y = norm_ref(xs[[0, 3, 6, 7]], None, w, 1e-6)
        within(r.y[[0, 3, 6, 7]], y, (ROUND[dtype] + 2.0 ** -14) * y.abs(), "y")


def norm_backward_ref(dy, s, rstd, w, dsum):
    g, r = d(dy) * d(w)[..., None, :], d(rstd)[..., None]
    along = (g * d(s)).mean(dim=-1, keepdim=True)
    dx = r * (g - d(s) * r * r * along) + (0 if dsum is None else d(dsum))
    return dx, (d(dy) * d(s) * r).sum(dim=-2)


@pytest.mark.parametrize("groups,rows,dim", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("with_dsum", [False, True])
def test_rmsnorm_backward(groups, rows, dim, dtype, with_dsum):
    s = randn(11, norm_shape(groups, rows, dim), 2.0, dtype)
    dy = randn(12, norm_shape(groups, rows, dim), 0.1, dtype)
    dsum = randn(13, norm_shape(groups, rows, dim), 0.1, dtype) if with_dsum else None
    w = 1 + randn(14, norm_shape(groups, dim), 0.2, F32)
    rstd = (s.float().square().mean(dim=-1) + 1e-6).rsqrt() if dim else None
    dx, dw = ops.rmsnorm_backward(dy, s, rstd, w, dsum=dsum)
    if rows == 0 or groups == 0:
        assert dx.shape == s.shape and (dw == 0).all()
        return
    ref_dx, ref_dw = norm_backward_ref(dy, s, rstd, w, dsum)
    g = d(dy).abs() * d(w).abs()[..., None, :]
    r = d(rstd)[..., None]
    size = r * (g + d(s).abs() * r * r * (g * d(s).abs()).mean(dim=-1, keepdim=True))
    size = size + (0 if dsum is None else d(dsum).abs())
    within(dx, ref_dx, ROUND[dtype] * ref_dx.abs() + ((dim + 16) * 2.0 ** -24 + 2.0 ** -20) * size, "dx")
    mag = (d(dy) * d(s) * r).abs().sum(dim=-2)
    within(dw, ref_dw, (rows + 16) * 2.0 ** -23 * mag, "dweight")
    dx2, none = ops.rmsnorm_backward(dy, s, rstd, w, dsum=dsum, want_dweight=False)
    assert none is None and torch.equal(dx, dx2)
    dx3, dw3 = ops.rmsnorm_backward(dy, s, rstd, w, dsum=dsum)
    assert torch.equal(dx, dx3) and torch.equal(dw, dw3)


# widths on both sides of the lanes that take a row, many rows, and counts that leave a last set in part
@pytest.mark.parametrize("groups,rows,dim", [(1, 1237, 8), (1, 700, 64), (3, 301, 72), (1, 2001, 128), (2, 777, 136),
                                             (144, 10, 256), (1, 650, 264), (1, 621, 512), (1, 613, 520),
                                             (5, 131, 784), (1, 609, 1024), (1, 615, 1032), (1, 640, 2048)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,e4m3", [(False, False), (True, False), (True, True)])
def test_many_short_rows(groups, rows, dim, dtype, residual, e4m3):
    test_rmsnorm(groups, rows, dim, dtype, residual, e4m3, not e4m3)
    if not residual:
        test_quantize_rows(groups, rows, dim, dtype)


@pytest.mark.parametrize("groups,rows,dim", [(1, 1237, 8), (1, 700, 32), (3, 301, 72), (1, 2001, 128), (2, 777, 136),
                                             (7, 33, 256), (1, 650, 264), (1, 621, 512), (1, 613, 520),
                                             (5, 131, 784), (1, 609, 1024), (80, 3, 64), (1, 3000, 264)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("with_dsum", [False, True])
def test_many_short_rows_backward(groups, rows, dim, dtype, with_dsum):
    test_rmsnorm_backward(groups, rows, dim, dtype, with_dsum)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 256, 784])
def test_many_short_rows_with_extremes_and_strides(dtype, dim):
    """Rows cut from wider ones, groups woven row by row, a shared weight, the stream updated in place; rows
    of zeros, of NaN and infinity and of the type's ends among them, each of which stays in its row."""
    rows, groups = 300, 4
    wide = randn(131, (rows, groups, dim + 16), 1.0, dtype)
    x = wide[:, :, 8:8 + dim].permute(1, 0, 2)
    w = (1 + randn(132, (1, dim), 0.1, F32)).expand(groups, dim)
    own = randn(133, (groups, rows, dim), 1.0, dtype)
    before, rest = own.clone(), wide.clone()
    r = ops.rmsnorm(x, w, residual=own, sum_out=own)
    check_norm(r, x, before, w, 1e-6, False, False)
    assert torch.equal(rest, wide)
    x = x.clone()
    x[0, 5], x[1, 6, 3], x[2, 7, 0] = 0.0, float("nan"), float("inf")
    x[3, 8] *= 1e-38
    x[0, 9] = torch.finfo(dtype).max
    q, s = ops.quantize_rows(x)
    y = ops.rmsnorm(x, w, e4m3=True)
    bad = torch.zeros(groups, rows, dtype=torch.bool, device="cuda")
    bad[1, 6] = bad[2, 7] = True
    for scale in (s, y.scale):
        assert torch.equal(~torch.isfinite(scale[bad]), torch.ones(2, dtype=torch.bool, device="cuda"))
    assert torch.isfinite(s[~bad]).all() and torch.isfinite(q.float()[~bad]).all()
    few_q, few_s = ops.quantize_rows(x[:, 4:10].contiguous())  # the same rows by the kernel for a few
    assert torch.equal(few_s.isnan(), s[:, 4:10].isnan())
    assert torch.equal(torch.nan_to_num(few_s), torch.nan_to_num(s[:, 4:10]))
    assert torch.equal(torch.nan_to_num(few_q.float()), torch.nan_to_num(q.float()[:, 4:10]))


def test_rmsnorm_gradients_are_those_of_the_forward():
    """Against central differences of the definition in 64 bits, along random directions."""
    rows, dim, eps = 5, 48, 1e-3
    x, w = randn(15, (rows, dim), 1.0, F32), 1 + randn(16, (dim,), 0.2, F32)
    c = randn(17, (rows, dim), 1.0, F32)
    r = ops.rmsnorm(x, w, eps=eps, keep=True)
    dx, dw = ops.rmsnorm_backward(c, x, r.rstd, w)

    def f(xx, ww):
        return (norm_ref(xx, None, ww, eps)[2] * d(c)).sum()

    h = 1e-5
    for seed in range(4):
        vx, vw = randn(20 + seed, (rows, dim), 1.0, F64), randn(30 + seed, (dim,), 1.0, F64)
        for got, diff in (((d(dx) * vx).sum(), f(d(x) + h * vx, d(w)) - f(d(x) - h * vx, d(w))),
                          ((d(dw) * vw).sum(), f(d(x), d(w) + h * vw) - f(d(x), d(w) - h * vw))):
            assert abs(got - diff / (2 * h)) < 1e-4


# rows that start anywhere in a 16-byte unit, enough of them to stream; a dimension past the kernels' widest
OFF_GRID = [(1, 1300, 257), (3, 300, 1001), (1, 650, 8191), (2, 700, 7), (1, 640, 1), (1, 700, 16383),
            (5, 200, 12), (1, 900, 4100), (1, 1000, 16378)]


@pytest.mark.parametrize("groups,rows,dim", OFF_GRID)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,e4m3", [(False, False), (True, True), (True, False)])
def test_many_rows_off_the_grid(groups, rows, dim, dtype, residual, e4m3):
    x = randn(121, norm_shape(groups, rows, dim), 2.0, dtype)
    res = randn(122, norm_shape(groups, rows, dim), 3.0, dtype) if residual else None
    w = 1 + randn(123, norm_shape(groups, dim), 0.2, F32)
    r = ops.rmsnorm(x, w, residual=res, eps=1e-5, e4m3=e4m3, keep=True)
    check_norm(r, x, res, w, 1e-5, e4m3, True)
    q, scale = ops.quantize_rows(x)
    ref = (d(x).abs().amax(dim=-1) / 448).clamp(min=2.0 ** -126)
    within(scale, ref, 2.0 ** -23 * ref, "scale")
    v = d(x) / ref[..., None]
    within(q, v, 2.0 ** -4 * v.abs() * (1 + 2.0 ** -20) + 2.0 ** -10, "q")


@pytest.mark.parametrize("groups,rows,dim", OFF_GRID)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("with_dsum", [False, True])
def test_many_rows_off_the_grid_backward(groups, rows, dim, dtype, with_dsum):
    test_rmsnorm_backward(groups, rows, dim, dtype, with_dsum)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("wide,cut,res_cut", [(264, 3, 3), (261, 0, 0), (264, 3, 2), (257, 1, 1)])
def test_many_strided_rows(dtype, wide, cut, res_cut):
    """Rows cut from wider ones, the residual at the same place in them or at another; the stream updated
    in place, and nothing beside it."""
    rows, groups, dim = 400, 3, 253
    x = randn(124, (rows, groups, wide), 1.0, dtype)[:, :, cut:cut + dim].permute(1, 0, 2)
    whole = randn(125, (rows, groups, wide), 1.0, dtype)
    res = whole[:, :, res_cut:res_cut + dim].permute(1, 0, 2)
    w = (1 + randn(126, (1, dim), 0.1, F32)).expand(groups, dim)
    before, beside = res.clone(), whole.clone()
    r = ops.rmsnorm(x, w, residual=res, sum_out=res, keep=True)
    check_norm(r, x, before, w, 1e-6, False, True)
    beside[:, :, res_cut:res_cut + dim] = whole[:, :, res_cut:res_cut + dim]
    assert torch.equal(beside, whole)
    dy = randn(127, (rows, groups, wide), 0.1, dtype)[:, :, cut:cut + dim].permute(1, 0, 2)
    dx, dw = ops.rmsnorm_backward(dy, res, r.rstd, w, dsum=x)
    ref_dx, ref_dw = norm_backward_ref(dy, res, r.rstd, w, x)
    g, rs = d(dy).abs() * d(w).abs()[..., None, :], d(r.rstd)[..., None]
    size = rs * (g + d(res).abs() * rs * rs * (g * d(res).abs()).mean(dim=-1, keepdim=True)) + d(x).abs()
    within(dx, ref_dx, ROUND[dtype] * ref_dx.abs() + ((dim + 16) * 2.0 ** -24 + 2.0 ** -20) * size, "dx")
    mag = (d(dy) * d(res) * rs).abs().sum(dim=-2)
    within(dw, ref_dw, (rows + 16) * 2.0 ** -23 * mag, "dweight")


# ---- quantize_rows --------------------------------------------------------------------------------
@pytest.mark.parametrize("groups,rows,dim", NORM_SHAPES + [(1, 3, 20000), (2, 2, 33333), (1, 2, 65536)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_rows(groups, rows, dim, dtype):
    x = randn(41, norm_shape(groups, rows, dim), 3.0, dtype)
    q, scale = ops.quantize_rows(x)
    assert q.shape == x.shape and q.dtype == E4M3 and scale.shape == x.shape[:-1]
    if rows == 0 or groups == 0:
        return
    ref = (d(x).abs().amax(dim=-1) / 448).clamp(min=2.0 ** -126)
    within(scale, ref, 2.0 ** -23 * ref, "scale")
    v = d(x) / ref[..., None]
    within(q, v, 2.0 ** -4 * v.abs() * (1 + 2.0 ** -20) + 2.0 ** -10, "q")


def test_quantize_rows_extremes_and_strides():
    x = randn(42, (8, 3, 40), 1.0, F32).permute(1, 0, 2)[:, :, 1:38]
    x[0, 1] = 0
    x[0, 2] *= 1e-42
    x[1, 3, 5] = float("nan")
    x[1, 4, 6] = float("-inf")
    q, scale = ops.quantize_rows(x)
    assert (q.float()[0, 1] == 0).all() and scale[0, 1] == 2.0 ** -126
    assert torch.isfinite(q.float()[0, 2]).all() and scale[0, 2] == 2.0 ** -126
    assert q.float()[1, 3].isnan().all() and scale[1, 3].isnan()
    assert scale[1, 4] == float("inf") and q.float()[1, 4, 6].isnan()
    assert (q.float()[1, 4, :6] == 0).all() and (q.float()[1, 4, 7:] == 0).all()
    ok = torch.ones(3, 8, dtype=torch.bool, device="cuda")
    ok[0, 1] = ok[0, 2] = ok[1, 3] = ok[1, 4] = False
    v = (d(x) / d(scale)[..., None])[ok]
    within(q[ok], v, 2.0 ** -4 * v.abs() * (1 + 2.0 ** -20) + 2.0 ** -10, "q")


def test_offsets_past_32_bits():
    """Rows that begin past 2^32 bytes and 2^31 elements."""
    rows, dim = 135000, 16384
    x = torch.zeros((rows, dim), dtype=BF16, device="cuda")
    x[-3:] = randn(43, (3, dim))
    q, scale = ops.quantize_rows(x)
    ref = d(x[-3:]).abs().amax(dim=-1) / 448
    within(scale[-3:], ref, 2.0 ** -23 * ref, "scale")
    v = d(x[-3:]) / ref[..., None]
    within(q[-3:], v, 2.0 ** -4 * v.abs() * (1 + 2.0 ** -20) + 2.0 ** -10, "q")
    assert (scale[:-3] == 2.0 ** -126).all()
    w = randn(44, (24, dim), 0.01)
    y, _ = ops.linear(x, w)
    u = d(x[-3:]) @ d(w).T
    mag = d(x[-3:]).abs() @ d(w).abs().T
    within(y[-3:], u, 2.0 ** -8 * u.abs() + sum_error(dim) * mag, "y")
    assert (y[:-3] == 0).all()


# ---- linear -----------------------------------------------------------------------------------------
# (groups, rows, k, n): single tokens, around the tile sizes 8, 16, 64, 128, 256, ragged and aligned
LINEAR_SHAPES = [(1, 1, 1, 1), (1, 1, 4096, 4096), (1, 1, 777, 1001), (1, 2, 64, 784), (5, 1, 256, 256),
                 (1, 4, 5000, 130), (1, 5, 256, 10), (1, 8, 1000, 264), (1, 9, 512, 1024),
                 (1, 16, 2048, 512), (1, 17, 100, 77), (3, 33, 784, 256), (1, 64, 256, 8192),
                 (1, 65, 1, 129), (1, 100, 16, 784), (12, 100, 256, 784), (1, 127, 65, 128),
                 (1, 128, 128, 128), (1, 129, 129, 257), (1, 200, 4096, 1024), (2, 300, 500, 333),
                 (1, 513, 64, 512), (1, 777, 500, 1001), (1, 1024, 784, 2048), (1, 2048, 1024, 2056),
                 (1, 4100, 256, 72), (1, 0, 64, 64), (0, 8, 64, 64)]


def operand(seed, shape, std, kind):
    x = randn(seed, shape, std)
    if kind == "e4m3":
        q, s = ops.quantize_rows(x)
        return q, s
    return x, None


def linear_ref(x, w, xs, ws, bias):
    x, w = d(x), d(w)
    if xs is not None:
        x, w = x * d(xs)[..., None], w * d(ws)[..., None]
    u, mag = x @ w.transpose(-1, -2), x.abs() @ w.abs().transpose(-1, -2)
    if bias is not None:
        u, mag = u + d(bias)[..., None, :], mag + d(bias).abs()[..., None, :]
    return u, mag


def check_linear(y, pre, x, w, xs, ws, bias, act, residual):
    u, mag = linear_ref(x, w, xs, ws, bias)
    err = sum_error(x.shape[-1]) * mag
    a = act64(act, u)
    out = a if residual is None else a + d(residual)
    within(y, out, ROUND[y.dtype] * out.abs() + 1.2 * err + 2.0 ** -18 * a.abs() + 1e-30, "y")
    if pre is not None:
        within(pre, u, 2.0 ** -8 * u.abs() + err + 1e-30, "pre")


@pytest.mark.parametrize("i", range(len(LINEAR_SHAPES)))
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("variant", [0, 1, 2])
def test_linear(i, kind, variant):
    groups, rows, k, n = LINEAR_SHAPES[i]
    act = ACTS[(i + 2 * variant) % 6]
    out_dtype = F32 if variant == 1 else BF16
    x, xs = operand(51, norm_shape(groups, rows, k), 1.0, kind)
    w, ws = operand(52, norm_shape(groups, n, k), k ** -0.5, kind)
    bias = randn(53, norm_shape(groups, n), 0.5, F32) if variant != 2 else None
    residual = randn(54, norm_shape(groups, rows, n), 1.0, out_dtype) if variant else None
    keep = variant != 1
    y, pre = ops.linear(x, w, bias, act=act, slope=SLOPE, residual=residual, x_scale=xs, w_scale=ws,
                        out_dtype=out_dtype, keep=keep)
    assert y.dtype == out_dtype and y.shape == norm_shape(groups, rows, n) and (pre is None) == (not keep)
    if groups and rows:
        check_linear(y, pre, x, w, xs, ws, bias, act, residual)
        again, _ = ops.linear(x, w, bias, act=act, slope=SLOPE, residual=residual, x_scale=xs,
                              w_scale=ws, out_dtype=out_dtype, keep=keep)
        assert torch.equal(y, again)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [1, 3, 24, 150, 600])
@pytest.mark.parametrize("k,n,cut", [(256, 320, 0), (256, 320, 3), (500, 333, 16), (123, 45, 1)])
def test_linear_strides_and_places(kind, rows, k, n, cut):
    """Operands cut from wider rows, groups woven row by row, an operand shared by the groups, and the
    residual updated in place."""
    groups = 3
    xw, _ = operand(61, (rows, groups, k + 32), 1.0, kind)
    x = xw[:, :, cut:cut + k].permute(1, 0, 2)
    w, _ = operand(62, (1, n, k), k ** -0.5, kind)
    w = w.expand(groups, n, k)
    xs = ws = None
    if kind == "e4m3":
        xs, ws = randn(63, (groups, rows), 0.1, F32).abs(), randn(64, (groups, n), 0.1, F32).abs()
    bias = randn(65, (1, n), 0.5, F32).expand(groups, n)
    wide = randn(66, (rows, groups, n + 7), 1.0)
    stream = wide[:, :, 5:5 + n].permute(1, 0, 2)
    before, rest = stream.clone(), wide.clone()
    y, pre = ops.linear(x, w, bias, act="silu", residual=stream, x_scale=xs, w_scale=ws, keep=True,
                        out=stream)
    assert y is stream
    check_linear(y, pre, x, w, xs, ws, bias, "silu", before)
    rest[:, :, 5:5 + n] = wide[:, :, 5:5 + n]
    assert torch.equal(rest, wide)  # nothing outside the output was written


@pytest.mark.parametrize("groups,rows,k,n", [(40, 300, 256, 520), (160, 100, 208, 264), (1, 20000, 256, 392),
                                             (24, 513, 64, 640), (1, 9000, 784, 512), (3, 7000, 240, 136)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("act,with_residual,keep", [("tanh", False, False), ("gelu", True, False),
                                                    ("none", True, True)])
def test_linear_short_sums(groups, rows, k, n, kind, act, with_residual, keep):
    """Many tiles of a few hundred k, one residual for every group, the stream updated in place."""
    x, xs = operand(161, norm_shape(groups, rows, k), 1.0, kind)
    w, ws = operand(162, norm_shape(groups, n, k), k ** -0.5, kind)
    bias = randn(163, norm_shape(groups, n), 0.5, F32)
    residual = None
    if with_residual:
        residual = randn(164, norm_shape(groups, rows, n))
        if groups > 1 and not keep:
            residual = residual[:1].expand(groups, rows, n)
    before = residual if residual is None or not keep else residual.clone()
    y, pre = ops.linear(x, w, bias, act=act, residual=residual, x_scale=xs, w_scale=ws, keep=keep,
                        out=residual if keep else None)
    check_linear(y, pre, x, w, xs, ws, bias, act, before)
    if not keep:
        again, _ = ops.linear(x, w, bias, act=act, residual=residual, x_scale=xs, w_scale=ws)
        assert torch.equal(y, again)


# One to four rows on both sides of the sizes at which another kernel takes them.
@pytest.mark.parametrize("groups,rows,k,n", [(1, 1, 64, 12352), (1, 2, 72, 12304), (1, 2, 72, 12280),
                                             (300, 1, 64, 48), (200, 2, 128, 72), (1, 2, 4112, 4096),
                                             (1, 3, 4112, 2048), (1, 4, 2050, 1023), (1, 4, 2050, 1029),
                                             (1, 2, 4099, 2053), (97, 4, 200, 33)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("apart", [0, 5])
def test_linear_few_rows(groups, rows, k, n, kind, apart):
    """Rows of x as they lie and with a gap that takes them off the 16-byte grid."""
    x, xs = operand(171, norm_shape(groups, rows, k + apart), 1.0, kind)
    x = x[..., :k]
    w, ws = operand(172, norm_shape(groups, n, k), k ** -0.5, kind)
    bias = randn(173, norm_shape(groups, n), 0.5, F32)
    residual = randn(174, norm_shape(groups, rows, n))
    y, pre = ops.linear(x, w, bias, act="gelu", residual=residual, x_scale=xs, w_scale=ws, keep=True)
    check_linear(y, pre, x, w, xs, ws, bias, "gelu", residual)
    again, _ = ops.linear(x, w, bias, act="gelu", residual=residual, x_scale=xs, w_scale=ws)
    assert torch.equal(y, again)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [1, 20, 300])
def test_linear_nan_and_infinity_stay_in_their_row_and_column(kind, rows):
    k, n = 200, 300
    x, xs = operand(71, (rows, k), 1.0, kind)
    w, ws = operand(72, (n, k), 0.1, kind)
    xf, wf = x.float(), w.float()
    xf[rows - 1, 5] = float("nan")
    wf[n - 1, 7] = float("nan")
    x, w = xf.to(x.dtype), wf.to(w.dtype)
    y, _ = ops.linear(x, w, act="gelu", x_scale=xs, w_scale=ws)
    assert y[rows - 1].isnan().all() and y[:, n - 1].isnan().all()
    assert torch.isfinite(y[:rows - 1, :n - 1]).all()


def backward_ref(dy, x, w, act, pre):
    du = d(dy) * (slope64(act, d(pre)) if act != "none" else 1.0)
    return du, du @ d(w), du.transpose(-1, -2) @ d(x), du.sum(dim=-2)


@pytest.mark.parametrize("i", range(len(LINEAR_SHAPES)))
@pytest.mark.parametrize("variant", [0, 1])
def test_linear_backward(i, variant):
    groups, rows, k, n = LINEAR_SHAPES[i]
    act = ACTS[(i + 3 * variant) % 6]
    dw_dtype = F32 if variant else BF16
    dy = randn(81, norm_shape(groups, rows, n), 0.1)
    x = randn(82, norm_shape(groups, rows, k))
    w = randn(83, norm_shape(groups, n, k), k ** -0.5)
    pre = randn(84, norm_shape(groups, rows, n), 1.5) if act != "none" else None
    dx, dw, db = ops.linear_backward(dy, x, w, act=act, slope=SLOPE, pre=pre, dw_dtype=dw_dtype)
    assert dx.dtype == BF16 and dw.dtype == dw_dtype and db.dtype == F32
    if rows == 0 or groups == 0:
        assert (dw == 0).all() and (db == 0).all() and dw.shape == w.shape
        return
    du, rx, rw, rb = backward_ref(dy, x, w, act, pre)
    delta = 0 if act == "none" else 2.0 ** -8 + 2.0 ** -17
    size = d(dy).abs()  # (the slopes stay below 1.2)
    mag = 1.2 * size @ d(w).abs()
    within(dx, rx, 2.0 ** -8 * rx.abs() + (delta + sum_error(n)) * mag + 1e-30, "dx")
    mag = 1.2 * size.transpose(-1, -2) @ d(x).abs()
    within(dw, rw, ROUND[dw_dtype] * rw.abs() + (delta + sum_error(rows)) * mag + 1e-30, "dw")
    within(db, rb, (2.0 ** -17 + (rows + 16) * 2.0 ** -24) * 1.2 * size.sum(dim=-2), "db")
    only = ops.linear_backward(dy, x, w, act=act, slope=SLOPE, pre=pre, want_dx=False, want_db=False,
                               dw_dtype=dw_dtype)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
    only = ops.linear_backward(dy, x, w, act=act, slope=SLOPE, pre=pre, want_dw=False)
    assert only[1] is None and torch.equal(only[0], dx) and torch.equal(only[2], db)


@pytest.mark.parametrize("rows,k,n,cut", [(150, 256, 320, 0), (150, 256, 320, 3), (40, 130, 77, 1)])
def test_linear_backward_strides(rows, k, n, cut):
    groups = 3
    dy = randn(91, (rows, groups, n + 16), 0.1)[:, :, cut:cut + n].permute(1, 0, 2)
    pre = randn(92, (rows, groups, n + 16))[:, :, cut:cut + n].permute(1, 0, 2)
    x = randn(93, (1, rows, k)).expand(groups, rows, k)
    w = randn(94, (1, n, k + 5), k ** -0.5)[:, :, cut:cut + k].expand(groups, n, k)
    dx, dw, db = ops.linear_backward(dy, x, w, act="silu", pre=pre)
    _, rx, rw, rb = backward_ref(dy, x, w, "silu", pre)
    size = 1.2 * d(dy).abs()
    delta = 2.0 ** -8 + 2.0 ** -17
    within(dx, rx, 2.0 ** -8 * rx.abs() + (delta + sum_error(n)) * (size @ d(w).abs()), "dx")
    within(dw, rw, 2.0 ** -8 * rw.abs()
           + (delta + sum_error(rows)) * (size.transpose(-1, -2) @ d(x).abs()), "dw")
    within(db, rb, (2.0 ** -17 + (rows + 16) * 2.0 ** -24) * size.sum(dim=-2), "db")


@pytest.mark.parametrize("rows,k,n,cut", [(150, 256, 320, 3), (40, 130, 77, 0), (700, 129, 250, 1), (1, 33, 9, 1),
                                          (3, 100, 100, 0)])
@pytest.mark.parametrize("groups", [1, 4])
def test_linear_backward_without_activation(rows, k, n, cut, groups):
    """dy off the 16-byte grid, operands that the groups share, and every choice of results: the same bits."""
    dy = randn(181, (groups, rows, n + 5), 0.1)[:, :, cut:cut + n]
    x = randn(182, (1, rows, k + 3))[:, :, cut:cut + k].expand(groups, rows, k)
    w = randn(183, (1, n, k + 3), k ** -0.5)[:, :, :k].expand(groups, n, k)
    dx, dw, db = ops.linear_backward(dy, x, w)
    _, rx, rw, rb = backward_ref(dy, x, w, "none", None)
    within(dx, rx, 2.0 ** -8 * rx.abs() + sum_error(n) * (d(dy).abs() @ d(w).abs()), "dx")
    within(dw, rw, 2.0 ** -8 * rw.abs() + sum_error(rows) * (d(dy).abs().transpose(-1, -2) @ d(x).abs()), "dw")
    within(db, rb, (rows + 16) * 2.0 ** -24 * d(dy).abs().sum(dim=-2), "db")
    for i in range(1, 7):
        want = [bool(i & 1), bool(i & 2), bool(i & 4)]
        got = ops.linear_backward(dy, x, w, want_dx=want[0], want_dw=want[1], want_db=want[2])
        for on, a, b in zip(want, got, (dx, dw, db)):
            assert (a is None) if not on else torch.equal(a, b)


@pytest.mark.parametrize("act", ACTS)
def test_linear_gradients_are_those_of_the_forward(act):
    """Against central differences of the definition in 64 bits along random directions: within the
    bf16 rounding of deltas and results, 2^-7 of the sum of magnitudes' root over the terms."""
    rows, k, n = 24, 40, 56
    x, w, b = randn(95, (rows, k)), randn(96, (n, k), k ** -0.5), randn(97, (n,), 0.3, F32)
    c = randn(98, (rows, n), 0.5)
    u = d(x) @ d(w).T + d(b)
    pre = u.to(BF16)
    if act in ("relu", "lrelu"):  # no kinks within a step of the differences
        pre = torch.where(pre.abs() < 1e-2, torch.full_like(pre, 0.05), pre)
    dx, dw, db = ops.linear_backward(c, x, w, act=act, slope=SLOPE, pre=pre)
    shift = d(pre) - u  # the differences are taken at the pre-activations that were kept

    def f(xx, ww, bb):
        return (act64(act, xx @ ww.T + bb + shift) * d(c)).sum()

    h = 1e-6
    at = [d(x), d(w), d(b)]
    for seed in range(3):
        for j, got in enumerate((dx, dw, db)):
            v = randn(100 + 10 * seed + j, at[j].shape, 1.0, F64)
            hi = [t + h * v if q == j else t for q, t in enumerate(at)]
            lo = [t - h * v if q == j else t for q, t in enumerate(at)]
            diff = (f(*hi) - f(*lo)) / (2 * h)
            size = (d(got) * v).square().sum().sqrt()
            assert abs((d(got) * v).sum() - diff) <= 2.0 ** -7 * size + 1e-6


@pytest.mark.parametrize("groups,rows,k,n", [(1, 4, 64, 16), (2, 300, 500, 333), (1, 777, 784, 256),
                                             (1, 5000, 96, 64)])
@pytest.mark.parametrize("dx_dtype,dw_dtype", [(F32, F32), (F32, BF16), (BF16, F32)])
def test_linear_backward_result_types(groups, rows, k, n, dx_dtype, dw_dtype):
    """Without an activation the deltas are exact, and fp32 gradients as near as fp32 sums; a gradient's
    values do not depend on whether the other is asked for."""
    dy, x = randn(111, norm_shape(groups, rows, n), 0.1), randn(112, norm_shape(groups, rows, k))
    w = randn(113, norm_shape(groups, n, k), k ** -0.5)
    kw = dict(dx_dtype=dx_dtype, dw_dtype=dw_dtype)
    dx, dw, db = ops.linear_backward(dy, x, w, **kw)
    assert dx.dtype == dx_dtype and dw.dtype == dw_dtype
    _, rx, rw, rb = backward_ref(dy, x, w, "none", None)
    within(dx, rx, ROUND[dx_dtype] * rx.abs() + sum_error(n) * (d(dy).abs() @ d(w).abs()), "dx")
    within(dw, rw, ROUND[dw_dtype] * rw.abs()
           + sum_error(rows) * (d(dy).abs().transpose(-1, -2) @ d(x).abs()), "dw")
    within(db, rb, (rows + 16) * 2.0 ** -24 * d(dy).abs().sum(dim=-2), "db")
    assert torch.equal(ops.linear_backward(dy, x, w, want_dw=False, **kw)[0], dx)
    assert torch.equal(ops.linear_backward(dy, x, w, want_dx=False, **kw)[1], dw)


@pytest.mark.parametrize("k", [1024, 8192])
def test_linear_sums_in_fp32_stay_near_64_bits(k):
    """The tensor cores truncate; fp32 results add their sums over 512 k in registers. Relative error in
    the 2-norm: below 2^-20, whatever k."""
    x, w = randn(114, (300, k)), randn(115, (200, k), k ** -0.5)
    u = d(x) @ d(w).T
    for rows in (300, 20):
        y, _ = ops.linear(x[:rows], w, out_dtype=F32)
        assert (d(y) - u[:rows]).norm() < 2.0 ** -20 * u[:rows].norm()


# ---- streams, graphs, refusals ------------------------------------------------------------------------
def _block(x, stream, w):
    r = ops.rmsnorm(x, w["g"], residual=stream, e4m3=True)
    a, _ = ops.linear(r.y, w["w1"], w["b1"], act="gelu", x_scale=r.scale, w_scale=w["s1"])
    q, s = ops.quantize_rows(a)
    return ops.linear(q, w["w2"], w["b2"], residual=r.sum, x_scale=s, w_scale=w["s2"])[0]


def _block_weights(dim, hidden):
    w = {"g": 1 + randn(1, (dim,), 0.1, F32), "b1": randn(2, (hidden,), 0.1, F32),
         "b2": randn(3, (dim,), 0.1, F32)}
    w["w1"], w["s1"] = ops.quantize_rows(randn(4, (hidden, dim), dim ** -0.5))
    w["w2"], w["s2"] = ops.quantize_rows(randn(5, (dim, hidden), hidden ** -0.5))
    return w


@pytest.mark.parametrize("rows", [1, 40, 700])
def test_calls_on_streams_and_in_a_graph(rows):
    dim, hidden = 256, 520
    w = _block_weights(dim, hidden)
    x, stream = randn(6, (rows, dim)), randn(7, (rows, dim))
    want = _block(x, stream, w)
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            outs.append([_block(x, stream, w) for _ in range(5)])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for out in outs for o in out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _block(x, stream, w)
    x.copy_(randn(8, (rows, dim)))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, _block(x, stream, w)) and not torch.equal(got, want)
    L.lipz_operator_status()


def test_refusals_launch_nothing():
    x, w = randn(1, (4, 64)), randn(2, (8, 64))
    g = torch.ones(64, device="cuda")
    q, s = ops.quantize_rows(x)
    bad = [
        lambda: ops.rmsnorm(x, g.to(BF16)), lambda: ops.rmsnorm(x, g[:63]),
        lambda: ops.rmsnorm(x.half(), g), lambda: ops.rmsnorm(x.cpu(), g),
        lambda: ops.rmsnorm(x, g, residual=x.float()), lambda: ops.rmsnorm(x, g, eps=-1.0),
        lambda: ops.rmsnorm(x, g, sum_out=x), lambda: ops.rmsnorm(x.t(), g[:4]),
        lambda: ops.rmsnorm(randn(3, (1, 16385)), torch.ones(16385, device="cuda")),
        lambda: ops.rmsnorm_backward(x, x, s[:3], g), lambda: ops.rmsnorm_backward(None, x, s, g),
        lambda: ops.quantize_rows(q), lambda: ops.quantize_rows(x[0]),
        lambda: ops.linear(x, w[:, :63]), lambda: ops.linear(x, w, act="swish"),
        lambda: ops.linear(x, w, out_dtype=torch.float16), lambda: ops.linear(x, q),
        lambda: ops.linear(q, q, x_scale=s), lambda: ops.linear(x, w, x_scale=s, w_scale=s),
        lambda: ops.linear(x, w, residual=x), lambda: ops.linear(x, w, torch.ones(7, device="cuda")),
        lambda: ops.linear(x.float(), w.float()), lambda: ops.linear(x, w, out=x),
        lambda: ops.linear(x, w, out=torch.empty(1, 8, dtype=BF16, device="cuda").expand(4, 8)),
        lambda: ops.linear_backward(x, x, w, act="gelu"), lambda: ops.linear_backward(x, x, w),
        lambda: ops.linear_backward(randn(4, (4, 8)), x, None),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(L.LipzError) as e:
            f()
        assert e.value.code == L.LIPZ_ERR_INVALID, i
    torch.cuda.synchronize()
