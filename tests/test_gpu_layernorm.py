"""Layer norm, forward (with its sum kept in 8 bits) and backward, against the definition in 64 bits.

Tolerances, element by element. A chain of fp32 additions over a row is at most 80 long (32 elements of a thread, five
steps over a warp, up to 32 warps, and what joins them), so the mean is off by up to delta = 80 2^-24 mean|s| and the
rounding of s itself, and the variance by 90 2^-24 of its value and 2 delta times the deviation: with q = delta rstd,
rstd is off by rel = 90 2^-24 + q + q^2 + 2^-22 of its value, and (s - mean) rstd by rel of its size, q, and the
roundings of s and of the products. The result's own rounding is half a unit: eps / 2 of its value.
"""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_1811_12843_gb300 as L
    from paper_1811_12843_gb300 import operators as ops
    from test_gpu_checkpoints import check_blocks
    from test_gpu_operators import d, norm_shape, randn, within

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


# one element, widths around a warp's vectors and a block's, ragged widths, the widest
NORM_SHAPES = [(1, 1, 1), (1, 1, 4096), (1, 3, 7), (1, 5, 64), (1, 37, 256), (3, 11, 257), (1, 9, 784),
               (2, 400, 1000), (1, 700, 2056), (1, 6, 4104), (1, 320, 8192), (2, 3, 8191), (1, 330, 16384),
               (1, 4, 16383), (144, 100, 256), (1, 1, 16384), (1, 0, 64), (0, 4, 64)]
# rows that start anywhere in a 16-byte unit, many of them; a dimension past the widest that is taken in units
OFF_GRID = [(1, 1300, 257), (3, 300, 1001), (1, 650, 8191), (2, 700, 7), (1, 640, 1), (1, 700, 16383),
            (5, 200, 12), (1, 900, 4100), (1, 1000, 16378), (1, 1300, 33), (1, 700, 8183), (1, 620, 8185), (3, 333, 505),
            (2, 900, 506), (144, 9, 77), (700, 1, 129), (1, 3001, 1537), (90, 8, 300)]


def norm64(x, residual, weight, bias, eps):
    s = d(x) if residual is None else d(x) + d(residual)
    mean = s.mean(dim=-1)
    off = s - mean[..., None]
    rstd = (off.square().mean(dim=-1) + eps).rsqrt()
    h = off * rstd[..., None]
    y = h * d(weight)[..., None, :]
    return s, mean, rstd, h, y if bias is None else y + d(bias)[..., None, :]


def check(r, x, residual, weight, bias, eps, e4m3=False, keep=False):
    s, mean, rstd, h, y = norm64(x, residual, weight, bias, eps)
    half = torch.finfo(x.dtype).eps / 2
    delta = 80 * 2.0 ** -24 * s.abs().mean(dim=-1) + 2.0 ** -24 * s.abs().amax(dim=-1)
    q = delta * rstd
    rel = 90 * 2.0 ** -24 + q + q * q + 2.0 ** -22
    b = torch.zeros_like(d(weight)) if bias is None else d(bias)
    tol = d(weight).abs()[..., None, :] * (h.abs() * rel[..., None] + q[..., None] +
                                           2.0 ** -23 * s.abs() * rstd[..., None])
    tol = tol + 2.0 ** -22 * (y.abs() + b.abs()[..., None, :])
    if e4m3:
        off = tol.amax(dim=-1)
        scale = (y.abs().amax(dim=-1) / 448).clamp(min=2.0 ** -126)
        within(r.scale, scale, off / 448 + 2.0 ** -22 * scale, "scale")
        v = y / scale[..., None]
        within(r.y, v, 2.0 ** -4 * v.abs() + 2.0 ** -10 + 1.07 * (tol + off[..., None]) / scale[..., None] +
               2.0 ** -20 * v.abs(), "y")
    else:
        assert r.scale is None
        within(r.y, y, half * y.abs() + (1 + half) * tol + 1e-37, "y")
    if residual is None:
        assert r.sum is x
    else:
        within(r.sum, s, half * s.abs() * (1 + 2.0 ** -15), "sum")
    if keep:
        # (fp32 numbers below 2^-126 lie 2^-149 apart, whatever their size)
        within(r.mean, mean, delta + 2.0 ** -24 * mean.abs() + 2.0 ** -149, "mean")
        within(r.rstd, rstd, rel * rstd, "rstd")
    else:
        assert r.mean is None and r.rstd is None
    if keep == "int8":
        check_blocks(r.kept, r.sum, "kept")
    else:
        assert r.kept is None


def inputs(groups, rows, dim, dtype, residual, bias, seed=1):
    x = (randn(seed, norm_shape(groups, rows, dim), 2.0, F32) + 0.7).to(dtype)
    res = randn(seed + 1, norm_shape(groups, rows, dim), 3.0, dtype) if residual else None
    w = 1 + randn(seed + 2, norm_shape(groups, dim), 0.2, F32)
    b = randn(seed + 3, norm_shape(groups, dim), 0.5, F32) if bias else None
    return x, res, w, b


FORWARD = [(False, False, True, True), (True, True, False, True), (True, False, "int8", False),
           (False, True, "int8", True), (True, True, "int8", True)]


@pytest.mark.parametrize("groups,rows,dim", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,e4m3,keep,bias", FORWARD)
def test_layernorm(groups, rows, dim, dtype, residual, e4m3, keep, bias):
    x, res, w, b = inputs(groups, rows, dim, dtype, residual, bias)
    r = ops.layernorm(x, w, b, residual=res, eps=1e-5, e4m3=e4m3, keep=keep)
    if rows == 0 or groups == 0:
        assert r.y.shape == x.shape
        return
    check(r, x, res, w, b, 1e-5, e4m3, keep)


SHORT = [(1, 1237, 8), (1, 700, 64), (3, 301, 72), (1, 2001, 128), (2, 777, 136), (144, 10, 256), (1, 650, 264),
         (1, 621, 512), (1, 613, 520), (5, 131, 784), (1, 609, 1024), (1, 615, 1032), (1, 640, 2048), (1, 650, 4096)]


@pytest.mark.parametrize("groups,rows,dim", SHORT)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,e4m3,keep,bias", FORWARD)
def test_many_rows(groups, rows, dim, dtype, residual, e4m3, keep, bias):
    test_layernorm(groups, rows, dim, dtype, residual, e4m3, keep, bias)


@pytest.mark.parametrize("groups,rows,dim", OFF_GRID)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,e4m3,keep,bias", FORWARD)
def test_many_rows_off_the_grid(groups, rows, dim, dtype, residual, e4m3, keep, bias):
    test_layernorm(groups, rows, dim, dtype, residual, e4m3, keep, bias)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [256, 250, 6000])
@pytest.mark.parametrize("rows", [33, 400])
def test_strides_and_places(dtype, dim, rows):
    """Rows cut from wider ones off the 16-byte grid, groups woven row by row, a shared residual, weight and bias,
    the residual stream updated in place, and nothing beside it."""
    groups = 4
    wide = randn(4, (rows, groups, dim + 5), 1.0, dtype)
    x = wide[:, :, 3:3 + dim].permute(1, 0, 2)
    res = randn(5, (1, rows, dim), 1.0, dtype).expand(groups, rows, dim)
    w = (1 + randn(6, (1, dim), 0.1, F32)).expand(groups, dim)
    b = randn(7, (1, dim), 0.1, F32).expand(groups, dim)
    before = wide.clone()
    for e4m3 in (False, True):
        check(ops.layernorm(x, w, b, residual=res, e4m3=e4m3, keep="int8"), x, res, w, b, 1e-5, e4m3, "int8")
    assert torch.equal(before, wide)
    for cut in (3, 2):  # the residual at the same place of a 16-byte unit, or at another
        whole = randn(8, (rows, groups, dim + 5), 1.0, dtype)
        own, beside = whole[:, :, cut:cut + dim].permute(1, 0, 2), whole.clone()
        old = own.clone()
        r = ops.layernorm(x, w, b, residual=own, sum_out=own, keep="int8")
        assert r.sum is own
        check(r, x, old, w, b, 1e-5, False, "int8")
        beside[:, :, cut:cut + dim] = whole[:, :, cut:cut + dim]
        assert torch.equal(beside, whole)


def test_y_over_x_keeps_x():
    """The C call with y in x's buffer: the checkpoint is of x as it was."""
    for rows, dim in ((5, 64), (700, 253), (700, 256), (640, 4096)):
        x, _, w, b = inputs(1, rows, dim, BF16, False, True, seed=41)
        own, row = x.clone(), -(-dim // 16) * 16
        data = torch.zeros(rows, row, device="cuda", dtype=torch.int8)
        scale = torch.zeros(rows, row // 16, device="cuda", dtype=torch.uint8)
        a = L.lipz_layernorm_args()
        a.struct_size, a.eps, a.groups, a.rows, a.dim = L.ctypes.sizeof(a), 1e-5, 1, rows, dim
        a.x = a.y = L.lipz_mat(own.data_ptr(), 0, dim, L.LIPZ_BF16, 0)
        a.weight, a.bias = L.lipz_vec(w.data_ptr(), 0), L.lipz_vec(b.data_ptr(), 0)
        a.kept = L.lipz_blocks(data.data_ptr(), 0, row, scale.data_ptr(), 0, row // 16)
        L.lipz_layernorm(a, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(own, ops.layernorm(x, w, b).y)
        check_blocks(ops.Checkpoint(data[:, :dim], scale), x)
        assert (data[:, dim:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [7, 900])
@pytest.mark.parametrize("dim,cut", [(77, 3), (256, 8), (301, 1), (509, 5), (1001, 7), (4099, 2), (2000, 16)])
def test_nan_beside_the_rows_stays_there(dtype, rows, dim, cut):
    """Rows cut from wider ones whose other columns are NaN: the bits of the same rows by themselves."""
    def cut_from(t):
        wide = torch.full((rows, dim + 32), float("nan"), device="cuda", dtype=dtype)
        wide[:, cut:cut + dim] = t
        return wide[:, cut:cut + dim], wide

    x, res, w, b = inputs(1, rows, dim, dtype, True, True, seed=31)
    dy = randn(36, (rows, dim), 0.1, dtype)
    (xc, _), (rc, _), (dc, _) = cut_from(x), cut_from(res), cut_from(dy)
    for e4m3 in (False, True):
        r = ops.layernorm(xc, w, b, residual=rc, e4m3=e4m3, keep="int8")
        check(r, x, res, w, b, 1e-5, e4m3, "int8")
    own, wide = cut_from(res)
    got = ops.layernorm(xc, w, b, residual=own, sum_out=own, keep=True)
    assert torch.equal(own, r.sum)
    assert wide[:, :cut].isnan().all() and wide[:, cut + dim:].isnan().all()
    back = ops.layernorm_backward(dc, own, got.mean, got.rstd, w, dsum=rc)
    check_backward(back, dy, r.sum, got.mean, got.rstd, w, res)
    back = ops.layernorm_backward(dc, r.kept, got.mean, got.rstd, w, dsum=rc)
    check_backward(back, dy, ops.restore_rows(r.kept, out_dtype=F32), got.mean, got.rstd, w, res)
    check_blocks(ops.checkpoint_rows(xc), x)


def test_rows_behind_two_gigaelements():
    """Offsets past 2^31: the last rows as by themselves."""
    rows, dim, last = 270000, 8192, 700
    x = torch.zeros(rows, dim, device="cuda", dtype=BF16)
    x[-last:] = randn(45, (last, dim), 1.0)
    w, b = 1 + randn(46, (dim,), 0.1, F32), randn(47, (dim,), 0.1, F32)
    tail = x[-last:].clone()
    few = ops.layernorm(tail, w, b, keep="int8")
    r = ops.layernorm(x, w, b, keep="int8")
    assert torch.equal(r.y[-last:], few.y) and torch.equal(r.mean[-last:], few.mean)
    assert torch.equal(r.kept.data[-last:], few.kept.data) and torch.equal(r.kept.scale[-last:], few.kept.scale)
    assert torch.equal(ops.restore_rows(r.kept)[-last:], ops.restore_rows(few.kept))
    c = ops.checkpoint_rows(x)
    assert torch.equal(c.data[-last:], few.kept.data)
    dx, dw, db = ops.layernorm_backward(x, r.kept, r.mean, r.rstd, w)  # (dy is zero but for the last rows)
    ref = ops.layernorm_backward(tail, few.kept, few.mean, few.rstd, w)
    assert torch.equal(dx[-last:], ref[0]) and (dx[:-last] == 0).all()
    for a, b2 in ((dw, ref[1]), (db, ref[2])):  # (summed in another order: 700 terms of order 1)
        assert (a - b2).abs().max() <= 2 * 800 * 2.0 ** -24 * 700


@pytest.mark.parametrize("rows", [9, 700])
@pytest.mark.parametrize("dim", [512, 509, 4096, 24])
def test_extreme_rows(rows, dim):
    """Rows of zeros and of one value, a far mean, subnormal and huge rows, NaN and infinity: each in its row."""
    x = randn(9, (rows, dim), 1.0, F32)
    x[0] = 0
    x[1] = 3.0
    x[2] += 1000.0
    x[3] *= 1e-41
    x[4] *= 1e15
    x[5, 7] = float("nan")
    x[6, dim - 1] = float("inf")
    w, b = 1 + randn(10, (dim,), 0.1, F32), randn(11, (dim,), 0.1, F32)
    ok = [i for i in range(rows) if i not in (5, 6)]
    for dtype in (F32, BF16):
        xs = x.to(dtype)
        for e4m3 in (False, True):
            r = ops.layernorm(xs, w, b, e4m3=e4m3, keep="int8")
            for t in (r.y.float(), r.mean, r.rstd) + ((r.scale,) if e4m3 else ()):
                assert torch.isfinite(t[ok]).all()
            assert r.y[5].float().isnan().all() and r.y[6].float().isnan().all()
            if e4m3:
                assert r.scale[5].isnan() and r.scale[6].isnan()
            few = xs[ok]
            check(ops.LayerNorm(r.y[ok], few, r.scale[ok] if e4m3 else None, r.mean[ok], r.rstd[ok], None),
                  few, None, w, b, 1e-5, e4m3, True)
            check_blocks(r.kept, xs)
            assert (r.y[0].float() * (r.scale[0] if e4m3 else 1)).sub(b).abs().max() < (0.04 if e4m3 else 0.002)
    # a row of one value: no variance, nothing but the bias (the mean is a product with 1 / dim: two roundings of 3,
    # times 1 / sqrt(1e-5) and the weight)
    y = ops.layernorm(x[1:2], w, b).y
    within(y, d(b)[None], 3 * 2.0 ** -23 * 317 * d(w).abs()[None] + 2.0 ** -23 * d(b).abs()[None], "one value")


def test_far_means_keep_the_variance():
    """Values 2^12 deviations from zero: a sum of squares would have lost the variance."""
    for rows in (4, 700):
        for dim in (256, 253, 4096):
            x = randn(12, (rows, dim), 1.0, F32) + 4096.0
            w, b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
            r = ops.layernorm(x, w, b, keep=True)
            check(r, x, None, w, b, 1e-5, False, True)
            rstd = norm64(x, None, w, b, 1e-5)[2]
            # (delta is a rounding or two of 4096 over log-depth sums in practice: 2^-24 80 4096 = 0.02 by the bound)
            within(r.rstd, rstd, 0.03 * rstd, "rstd")


# ---- backward
def backward64(dy, s, mean, rstd, w, dsum):
    off, r = d(s) - d(mean)[..., None], d(rstd)[..., None]
    g = d(dy) * d(w)[..., None, :]
    dx = r * (g - g.mean(dim=-1, keepdim=True) - off * r * r * (g * off).mean(dim=-1, keepdim=True))
    return dx + (0 if dsum is None else d(dsum)), (d(dy) * off * r).sum(dim=-2), d(dy).sum(dim=-2)


def check_backward(got, dy, s, mean, rstd, w, dsum):
    """(Chains of up to 100 additions along a row, of rows + 100 down the columns; s - mean is rounded once.)"""
    dx, dw, db = got
    ref_dx, ref_dw, ref_db = backward64(dy, s, mean, rstd, w, dsum)
    off, r = (d(s) - d(mean)[..., None]).abs(), d(rstd)[..., None]
    g = (d(dy) * d(w)[..., None, :]).abs()
    size = r * (g + g.mean(dim=-1, keepdim=True) + off * r * r * (g * off).mean(dim=-1, keepdim=True))
    size = size + (0 if dsum is None else d(dsum).abs())
    half, n = torch.finfo(dy.dtype).eps / 2, dy.shape[-2] + 100
    within(dx, ref_dx, half * ref_dx.abs() + 110 * 2.0 ** -24 * size + 1e-38, "dx")
    if dw is not None:
        within(dw, ref_dw, n * 2.0 ** -24 * (d(dy).abs() * off * r).sum(dim=-2) + 1e-38, "dweight")
    if db is not None:
        within(db, ref_db, n * 2.0 ** -24 * d(dy).abs().sum(dim=-2) + 1e-38, "dbias")


def backward_inputs(groups, rows, dim, dtype, with_dsum, seed=11):
    s = (randn(seed, norm_shape(groups, rows, dim), 2.0, F32) + 0.5).to(dtype)
    dy = randn(seed + 1, norm_shape(groups, rows, dim), 0.1, dtype)
    dsum = randn(seed + 2, norm_shape(groups, rows, dim), 0.1, dtype) if with_dsum else None
    w = 1 + randn(seed + 3, norm_shape(groups, dim), 0.2, F32)
    mean = s.float().mean(dim=-1)
    rstd = ((s.float() - mean[..., None]).square().mean(dim=-1) + 1e-5).rsqrt()
    return s, dy, dsum, w, mean, rstd


@pytest.mark.parametrize("groups,rows,dim", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("with_dsum", [False, True])
@pytest.mark.parametrize("kept", [False, True])
def test_layernorm_backward(groups, rows, dim, dtype, with_dsum, kept):
    s, dy, dsum, w, mean, rstd = backward_inputs(groups, rows, dim, dtype, with_dsum)
    given = s
    if kept:
        given = ops.checkpoint_rows(s)
        s = ops.restore_rows(given, out_dtype=F32)
    got = ops.layernorm_backward(dy, given, mean, rstd, w, dsum=dsum)
    if rows == 0 or groups == 0:
        assert got[0].shape == dy.shape and (got[1] == 0).all() and (got[2] == 0).all()
        return
    check_backward(got, dy, s, mean, rstd, w, dsum)
    for want in ((True, False), (False, True), (False, False)):
        some = ops.layernorm_backward(dy, given, mean, rstd, w, dsum=dsum, want_dweight=want[0], want_dbias=want[1])
        for a, b, wanted in zip(some, got, (True,) + want):
            assert torch.equal(a, b) if wanted else a is None
    if kept:  # rows at any byte
        whole = ops.Checkpoint(given.data.contiguous(), given.scale)
        check_backward(ops.layernorm_backward(dy, whole, mean, rstd, w, dsum=dsum), dy, s, mean, rstd, w, dsum)


@pytest.mark.parametrize("groups,rows,dim", SHORT + [(80, 3, 64), (1, 3000, 264)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("with_dsum", [False, True])
@pytest.mark.parametrize("kept", [False, True])
def test_many_rows_backward(groups, rows, dim, dtype, with_dsum, kept):
    test_layernorm_backward(groups, rows, dim, dtype, with_dsum, kept)


@pytest.mark.parametrize("groups,rows,dim", OFF_GRID)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("with_dsum", [False, True])
@pytest.mark.parametrize("kept", [False, True])
def test_many_rows_off_the_grid_backward(groups, rows, dim, dtype, with_dsum, kept):
    test_layernorm_backward(groups, rows, dim, dtype, with_dsum, kept)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [253, 256, 2056])
@pytest.mark.parametrize("rows", [21, 400])
def test_backward_strides(dtype, dim, rows):
    groups = 3

    def cut(seed, at):
        return randn(seed, (rows, groups, dim + 8), 0.5, dtype)[:, :, at:at + dim].permute(1, 0, 2)

    s, dy = cut(51, 3), cut(52, 3)
    w = (1 + randn(53, (1, dim), 0.1, F32)).expand(groups, dim)
    mean = s.float().mean(dim=-1)
    rstd = ((s.float() - mean[..., None]).square().mean(dim=-1) + 1e-5).rsqrt()
    for dsum in (cut(54, 3), cut(55, 2), randn(56, (1, rows, dim), 0.5, dtype).expand(groups, rows, dim)):
        check_backward(ops.layernorm_backward(dy, s, mean, rstd, w, dsum=dsum), dy, s, mean, rstd, w, dsum)
        kept = ops.checkpoint_rows(s)
        check_backward(ops.layernorm_backward(dy, kept, mean, rstd, w, dsum=dsum), dy,
                       ops.restore_rows(kept, out_dtype=F32), mean, rstd, w, dsum)


def test_backward_in_place():
    """The C call with dx in the place of dy, of s or of dsum."""
    for rows, dim in ((5, 64), (700, 253), (700, 256), (640, 4096), (3, 9000)):
        for place in ("dy", "s", "dsum"):
            s, dy, dsum, w, mean, rstd = backward_inputs(1, rows, dim, BF16, True, seed=61)
            want = ops.layernorm_backward(dy, s, mean, rstd, w, dsum=dsum)[0]
            a = L.lipz_layernorm_backward_args()
            a.struct_size, a.groups, a.rows, a.dim = L.ctypes.sizeof(a), 1, rows, dim
            t = dict(dy=dy, s=s, dsum=dsum)
            for name, v in t.items():
                setattr(a, name, L.lipz_mat(v.data_ptr(), 0, dim, L.LIPZ_BF16, 0))
            a.dx = L.lipz_mat(t[place].data_ptr(), 0, dim, L.LIPZ_BF16, 0)
            a.weight, a.mean, a.rstd = (L.lipz_vec(v.data_ptr(), 0) for v in (w, mean, rstd))
            assert L.lipz_layernorm_backward_workspace(a) == 0  # (no sums over rows are wanted)
            L.lipz_layernorm_backward(a, torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            assert torch.equal(t[place], want), (rows, dim, place)


def test_backward_of_rows_with_nan_and_infinity():
    """Each stays in its row of dx, and reaches the columns' sums."""
    for rows, dim in ((9, 64), (700, 253), (700, 512), (640, 4096)):
        s, dy, _, w, mean, rstd = backward_inputs(1, rows, dim, BF16, False, seed=71)
        dy[3, 5], s[4, 6] = float("nan"), float("inf")
        dx, dw, db = ops.layernorm_backward(dy, s, mean, rstd, w)
        ok = [i for i in range(rows) if i not in (3, 4)]
        assert torch.isfinite(dx[ok]).all() and dx[3].isnan().all() and not torch.isfinite(dx[4]).any()
        bad = torch.zeros(dim, dtype=torch.bool, device="cuda")
        bad[5] = True
        assert torch.equal(db.isnan(), bad)
        bad[6] = True
        assert torch.equal(~torch.isfinite(dw), bad)


def test_rows_so_small_that_rstd_squared_is_infinite():
    s, dy, _, w, _, _ = backward_inputs(1, 700, 256, F32, False, seed=81)
    for rows in (9, 700):
        t = s[:rows] * 2.0 ** -70
        mean = t.mean(dim=-1)
        rstd = (1 / (t.to(F64) - mean.to(F64)[:, None]).square().mean(dim=-1).sqrt()).float()
        got = ops.layernorm_backward(dy[:rows], t, mean, rstd, w)
        assert torch.isfinite(got[0]).all()
        check_backward(got, dy[:rows], t, mean, rstd, w, None)


def test_gradients_are_those_of_the_forward():
    """Against central differences of the definition in 64 bits, along random directions."""
    rows, dim, eps = 5, 48, 1e-3
    x, _, w, b = inputs(1, rows, dim, F32, False, True, seed=15)
    c = randn(19, (rows, dim), 1.0, F32)
    r = ops.layernorm(x, w, b, eps=eps, keep=True)
    got = ops.layernorm_backward(c, x, r.mean, r.rstd, w)

    def f(xx, ww, bb):
        return (norm64(xx, None, ww, bb, eps)[4] * d(c)).sum()

    h, at = 1e-5, [d(x), d(w), d(b)]
    for seed in range(4):
        for i, g in enumerate(got):
            v = randn(20 + 10 * i + seed, g.shape, 1.0, F64)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            assert abs((d(g) * v).sum() - (f(*up) - f(*down)) / (2 * h)) < 1e-4


# ---- together
def block(x, stream, p, keep8):
    """A pre-norm block's forward and backward; what it keeps in 8 bits, or as it is."""
    n = ops.layernorm(x, p["g"], p["beta"], residual=stream, keep="int8" if keep8 else True)
    h, pre = ops.linear(n.y, p["w1"], p["b1"], act="gelu", keep="int8" if keep8 else True)
    y = ops.linear(h, p["w2"], p["b2"])[0]
    ins, acts, total = ((ops.checkpoint_rows(n.y), ops.checkpoint_rows(h), n.kept) if keep8 else (n.y, h, n.sum))
    dh, dw2, db2 = ops.linear_backward(p["dy"], acts, p["w2"])
    dn, dw1, db1 = ops.linear_backward(dh, ins, p["w1"], act="gelu", pre=pre)
    dx, dg, dbeta = ops.layernorm_backward(dn, total, n.mean, n.rstd, p["g"], dsum=p["dy"])
    return [y, n.sum, dx, dg, dbeta, dw1, db1, dw2, db2]


def block_inputs(groups, rows, dim, hidden, seed=91):
    shape = (lambda *s: norm_shape(groups, *s))
    p = dict(g=1 + randn(seed, shape(dim), 0.1, F32), beta=randn(seed + 1, shape(dim), 0.1, F32),
             w1=randn(seed + 2, shape(hidden, dim), dim ** -0.5), b1=randn(seed + 3, shape(hidden), 0.1, F32),
             w2=randn(seed + 4, shape(dim, hidden), hidden ** -0.5), b2=randn(seed + 5, shape(dim), 0.1, F32),
             dy=randn(seed + 6, shape(rows, dim), 0.05))
    return randn(seed + 7, shape(rows, dim), 1.0), randn(seed + 8, shape(rows, dim), 1.0), p


@pytest.mark.parametrize("groups,rows,dim,hidden", [(1, 37, 100, 333), (5, 100, 256, 512), (1, 700, 784, 1001)])
def test_a_block_in_8_bits(groups, rows, dim, hidden):
    """The sum is the same, and y but for the order of its sums, which may move a rounding to bf16 (2^-8 of an element at
    most) of h or of y; gradients are off by what half a step of each block, 2^-7 of its largest at most and as good as
    random, does to them: below 2^-5 of a gradient's rms, as are bf16's own roundings."""
    x, stream, p = block_inputs(groups, rows, dim, hidden)
    whole, kept = block(x, stream, p, False), block(x, stream, p, True)
    assert torch.equal(whole[1], kept[1])
    assert (d(whole[0]) - d(kept[0])).square().mean().sqrt() <= 2.0 ** -8 * d(whole[0]).square().mean().sqrt()
    for a, b in zip(whole[2:], kept[2:]):
        assert a.shape == b.shape and a.dtype == b.dtype
        assert ((d(a) - d(b)).square().mean().sqrt() <= 2.0 ** -5 * d(a).square().mean().sqrt())


def test_a_block_in_a_graph_and_on_streams():
    """A captured step replayed on new inputs, two such graphs by turns, and two streams at once: the eager bits."""
    x, stream, p = block_inputs(3, 100, 256, 501)
    x2, stream2, p2 = block_inputs(3, 100, 256, 501, seed=191)
    want, want2 = block(x, stream, p, True), block(x2, stream2, p2, True)
    s = torch.cuda.Stream()
    graphs = []
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for args in ((x, stream, p), (x2, stream2, p2)):
            block(*args, True)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                out = block(*args, True)
            graphs.append((g, out))
    torch.cuda.synchronize()
    for _ in range(3):
        for g, out in graphs:
            g.replay()
    torch.cuda.synchronize()
    for (g, out), ref in zip(graphs, (want, want2)):
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
    x.copy_(x2), stream.copy_(stream2)
    for k in p:
        p[k].copy_(p2[k])
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(graphs[0][1], want2))
    t = torch.cuda.Stream()
    for u in (s, t):
        u.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = block(x, stream, p, True)
    with torch.cuda.stream(t):
        b = block(x2, stream2, p2, True)
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) and torch.equal(u, w) for u, v, w in zip(a, b, want2))


def test_refusals():
    x, res, w, b = inputs(1, 8, 64, BF16, True, True)
    r = ops.layernorm(x, w, b, residual=res, keep="int8")
    dy = randn(101, (8, 64), 0.1)
    bad = [
        (lambda: ops.layernorm(x, None, b), "weight must be given"),
        (lambda: ops.layernorm(x, w.bfloat16(), b), "weight has dtype"),
        (lambda: ops.layernorm(x, w, b[:63]), "bias has shape"),
        (lambda: ops.layernorm(x.half(), w, b), "dtype"),
        (lambda: ops.layernorm(x, w, b, residual=res.float()), "residual has dtype"),
        (lambda: ops.layernorm(x, w, b, sum_out=x), "sum_out needs"),
        (lambda: ops.layernorm(x, w, b, keep="int4"), "keep"),
        (lambda: ops.layernorm(x, w, b, eps=-1.0), "eps"),
        (lambda: ops.layernorm(x.clone().requires_grad_(True), w, b), "gradient"),
        (lambda: ops.layernorm(torch.zeros(2, 16385, device="cuda"), torch.ones(16385, device="cuda")), "dim"),
        (lambda: ops.layernorm_backward(dy, None, r.mean, r.rstd, w), "s must be given"),
        (lambda: ops.layernorm_backward(dy, r.sum, None, r.rstd, w), "mean must be given"),
        (lambda: ops.layernorm_backward(dy, r.sum.float(), r.mean, r.rstd, w), "s has dtype"),
        (lambda: ops.layernorm_backward(dy, r.kept.data, r.mean, r.rstd, w), "s has dtype"),
        (lambda: ops.layernorm_backward(dy, ops.Checkpoint(r.kept.data[:, :63], r.kept.scale), r.mean, r.rstd, w),
         "s has shape"),
        (lambda: ops.layernorm_backward(dy, r.sum, r.mean[:7], r.rstd, w), "mean has shape"),
    ]
    for f, what in bad:
        with pytest.raises(L.LipzError) as e:
            f()
        assert e.value.code == L.LIPZ_ERR_INVALID and what in str(e.value), (what, str(e.value))
