"""Activations in 8 bits: rows to checkpoints and back, the product that keeps its pre-activations so, and its
backward pass over them, against the definition.

A checkpoint is compared to the bit: its multiples and its bytes are whole numbers. The product's pre-activations are
fp32 results of the same call where there is no activation, so there the comparison is exact too; beside bf16 results
they are within half a step of their block (its largest over 127.5 at most) and the error of a sum of k products
(test_gpu_operators.py). A backward pass over checkpoints has the bits of one over the bf16 values that they stand for.
"""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_1811_12843_gb300 as L
    from paper_1811_12843_gb300 import operators as ops
    from test_gpu_operators import SLOPE, act64, backward_ref, d, norm_shape, randn, sum_error, within

ACTS = ["none", "relu", "lrelu", "tanh", "gelu", "silu"]
BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def blocks64(x):
    """x [.., columns] in 64 bits as (multiples, bytes, values): NaN blocks have the byte 255."""
    cols, n = x.shape[-1], -(-x.shape[-1] // 16)
    v = torch.nn.functional.pad(d(x), (0, n * 16 - cols)).unflatten(-1, (n, 16))
    top = v.abs().amax(dim=-1)
    bad = ~torch.isfinite(v).all(dim=-1)
    # top / 127.5 = m 2^e with m in [1/2, 1): 2^(e - 1) <= top / 127.5 < 2^e
    e = torch.frexp(torch.where(bad, torch.ones_like(top), top) / 127.5)[1].to(torch.int64)
    e = torch.where(top == 0, torch.full_like(e, -126), e).clamp(min=-126)
    unit = ((e + 1023) << 52).view(F64)[..., None]  # (2^e from its bits: torch.ldexp takes a power, which rounds)
    q = torch.round(v / unit)
    values = torch.where(bad[..., None], torch.full_like(q, float("nan")), q * unit)
    values = torch.where(values.abs() >= 2.0 ** 128, torch.sign(values) * float("inf"), values)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127)
    return q.flatten(-2)[..., :cols], byte, values.flatten(-2)[..., :cols], bad


def check_blocks(c, x, what="checkpoint"):
    """c is x's checkpoint, to the bit."""
    q, byte, values, bad = blocks64(x)
    assert c.data.dtype is torch.int8 and c.scale.dtype is torch.uint8
    assert c.data.shape == x.shape and c.scale.shape == byte.shape
    assert torch.equal(c.scale.to(torch.int64), byte), what
    ok = ~bad.repeat_interleave(16, dim=-1)[..., :x.shape[-1]]
    assert torch.equal(c.data.to(F64)[ok], q[ok]), what
    assert int(c.data.to(torch.int64).abs().max()) <= 127 if c.data.numel() else True


SHAPES = [(1, 1, 1), (1, 1, 4096), (1, 3, 7), (1, 5, 15), (1, 2, 16), (1, 33, 17), (1, 37, 500), (3, 11, 1001),
          (1, 700, 2056), (2, 9, 24), (144, 7, 256), (1, 2, 40001), (1, 0, 64), (0, 4, 64)]


@pytest.mark.parametrize("groups,rows,dim", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_to_checkpoints_and_back(groups, rows, dim, dtype):
    x = randn(1, norm_shape(groups, rows, dim), 2.0, dtype)
    c = ops.checkpoint_rows(x)
    check_blocks(c, x)
    y = ops.restore_rows(c)
    assert y.dtype is BF16 and torch.equal(d(y), blocks64(x)[2])
    assert torch.equal(ops.restore_rows(c, out_dtype=F32), y.float())
    whole = ops.Checkpoint(c.data.contiguous(), c.scale.contiguous())  # (rows at any byte)
    assert torch.equal(ops.restore_rows(whole), y)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [1001, 512])
def test_restored_activations(act, out_dtype, dim):
    """act of the values: within half a unit of the result's type, and in fp32 the hardware's exponential and
    reciprocal (2^-20, and 2^-21 times an exponent of up to 2 sqrt(2/pi) (8 + 0.0447 8^3) = 50). The reference's own
    1 + tanh is off by 2^-53 and more than that of nothing at all (u / 2 of it: 8 2^-53 covers it)."""
    x = randn(2, (65, dim), 3.0, F32).clamp(-8, 8)
    c = ops.checkpoint_rows(x)
    ref = act64(act, blocks64(x)[2])
    got = ops.restore_rows(c, act=act, slope=SLOPE, out_dtype=out_dtype)
    assert got.dtype is out_dtype
    rel = torch.finfo(out_dtype).eps / 2 + 2.0 ** -20 + 50 * 2.0 ** -21
    within(got, ref, rel * ref.abs() + 8 * 2.0 ** -53, act)


def test_extreme_rows():
    """Zeros, subnormals, the borders of a power of two, ties, the ends of the type, NaN and infinities."""
    x = torch.zeros(16, 40, device="cuda", dtype=F32)
    x[1] = randn(3, (40,), 1.0, F32) * 1e-39
    x[2] = 2.0 ** -149
    x[3, 5] = 127.5  # the next power of two
    x[4, 5] = torch.nextafter(torch.tensor(127.5), torch.tensor(0.0)).item()
    x[5, :16] = torch.arange(16, device="cuda") - 7.5  # ties, at a unit of 1 by the next element
    x[5, 15] = 127.0
    x[6] = torch.finfo(F32).max
    x[6, 20] = -127.0 * 2.0 ** 121
    x[7, 17] = float("nan")
    x[8, 0], x[8, 39] = float("inf"), -float("inf")
    x[9] = randn(4, (40,), 1.0, F32) * 2.0 ** 126
    x[10, ::2] = -0.0
    x[11] = torch.arange(40, device="cuda") * 2.0 ** -127  # ties of the smallest unit
    x[12, 3], x[12, 4] = float("nan"), float("inf")
    for dtype in (F32, BF16):
        for cols in (40, 33, 16):
            xs = x.to(dtype)[:, :cols].contiguous()
            c = ops.checkpoint_rows(xs)
            check_blocks(c, xs, (dtype, cols))
            y = ops.restore_rows(c)
            ref = blocks64(xs)[2]
            assert torch.equal(y.isnan(), ref.isnan()) and torch.equal(d(y).nan_to_num(0.0), ref.nan_to_num(0.0))


def test_bytes_of_any_value_are_read():
    """Byte 255 stands for NaN whatever the multiples are, and 0 for nothing."""
    q = torch.arange(-128, 128, device="cuda").to(torch.int8).reshape(8, 32)
    for byte in (0, 1, 100, 200, 249, 255):
        scale = torch.full((8, 2), byte, device="cuda", dtype=torch.uint8)
        y = ops.restore_rows(ops.Checkpoint(q, scale))
        if byte == 255:
            assert y.isnan().all()
        else:
            ref = d(q) * (2.0 ** (byte - 127) if byte else 0.0)
            assert torch.equal(d(y), torch.where(ref.abs() >= 2.0 ** 128, ref.sign() * float("inf"), ref))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [253, 256])
def test_strides_and_places(dtype, dim):
    """Rows cut from wider ones off the 16-byte grid, groups woven row by row, an input that the groups share."""
    rows, groups = 33, 4
    wide = randn(5, (rows, groups, dim + 5), 1.0, dtype)
    x = wide[:, :, 3:3 + dim].permute(1, 0, 2)
    c = ops.checkpoint_rows(x)
    check_blocks(c, x)
    check_blocks(ops.checkpoint_rows(x[:1].expand(groups, rows, dim)), x[:1].expand(groups, rows, dim))
    n = -(-dim // 16)
    data = torch.empty(rows, groups, dim + 7, device="cuda", dtype=torch.int8)[:, :, 5:5 + dim].permute(1, 0, 2)
    scale = torch.empty(rows, groups, n + 3, device="cuda", dtype=torch.uint8)[:, :, 1:1 + n].permute(1, 0, 2)
    data.copy_(c.data), scale.copy_(c.scale)
    assert torch.equal(ops.restore_rows(ops.Checkpoint(data, scale)), ops.restore_rows(c))
    one = ops.Checkpoint(c.data[:1].expand(groups, rows, dim), c.scale[:1].expand(groups, rows, n))
    assert torch.equal(ops.restore_rows(one), ops.restore_rows(ops.Checkpoint(c.data[:1], c.scale[:1])).expand(
        groups, rows, dim))


# ---- products
# one to four rows, a cluster's parts of k, rows that TMA does not take, each shape of tile, whole and ragged
LINEARS = [(1, 1, 256, 16), (1, 1, 4096, 4096), (1, 3, 513, 37), (1, 4, 512, 1000), (1, 2, 8, 9), (1, 37, 1000, 500),
           (1, 16, 4096, 512), (1, 5, 777, 61), (3, 100, 256, 512), (1, 300, 333, 257), (1, 513, 512, 1001),
           (2, 700, 64, 784), (1, 1300, 256, 2048), (1, 2048, 128, 4096), (17, 1, 300, 40), (1, 128, 2048, 8),
           (1, 0, 64, 32), (0, 3, 64, 32)]


def product(groups, rows, k, n, e4m3=False):
    shape = (lambda *s: norm_shape(groups, *s))
    x, w = randn(11, shape(rows, k), 1.0), randn(12, shape(n, k), k ** -0.5)
    b = randn(13, shape(n), 0.3, F32)
    xs = ws = None
    if e4m3:
        (x, xs), (w, ws) = ops.quantize_rows(x), ops.quantize_rows(w)
    u = d(x) @ d(w).transpose(-1, -2)
    size = d(x).abs() @ d(w).abs().transpose(-1, -2)
    if e4m3:
        f = d(xs)[..., None] * d(ws)[..., None, :]
        u, size = u * f, size * f
    return x, w, b, xs, ws, u + d(b)[..., None, :], size + d(b).abs()[..., None, :]


@pytest.mark.parametrize("groups,rows,k,n", LINEARS)
@pytest.mark.parametrize("e4m3", [False, True])
def test_linear_keeps_a_checkpoint(groups, rows, k, n, e4m3):
    x, w, b, xs, ws, u, size = product(groups, rows, k, n, e4m3)
    kw = dict(x_scale=xs, w_scale=ws)
    if rows == 0 or groups == 0:
        y, pre = ops.linear(x, w, b, keep="int8", **kw)
        assert pre.data.shape == u.shape and pre.scale.shape == u.shape[:-1] + (-(-n // 16),)
        return
    y, pre = ops.linear(x, w, b, out_dtype=F32, keep="int8", **kw)
    check_blocks(pre, y)
    for act, residual in (("gelu", None), ("silu", randn(14, u.shape, 1.0)), ("none", None)):
        y, pre = ops.linear(x, w, b, act=act, residual=residual, keep="int8", **kw)
        # (its sums are added up in other parts than without a checkpoint: gelu's and silu's slopes are below 1.13)
        ref = act64(act, u) + (0 if residual is None else d(residual))
        within(y, ref, 2.0 ** -8 * ref.abs() * (1 + 2.0 ** -7) + 1.13 * sum_error(k) * size * (1 + 2.0 ** -8) +
               2.0 ** -17 * act64(act, u).abs() * (1 + u.abs()), act)
        top = torch.nn.functional.pad(u.abs() + sum_error(k) * size, (0, -n % 16))
        top = top.unflatten(-1, (-(-n // 16), 16)).amax(dim=-1).repeat_interleave(16, dim=-1)[..., :n]
        within(ops.restore_rows(pre), u, top / 127.5 + sum_error(k) * size, act)


def test_a_checkpoint_of_nan_and_infinity_stays_in_its_row():
    """(Columns past the last one meet the row's infinity as 0 times infinity.)"""
    for rows, n in ((3, 37), (130, 37), (600, 300)):
        x, w = randn(15, (rows, 256), 1.0), randn(16, (n, 256), 0.1)
        x[1, 7] = float("nan")
        x[2, 9] = float("inf")
        y, pre = ops.linear(x, w, out_dtype=F32, keep="int8")
        check_blocks(pre, y)
        assert (pre.scale[1:3] == 255).all() and (pre.scale[0] != 255).all()


@pytest.mark.parametrize("rows,k,n", [(3, 256, 37), (40, 256, 300), (130, 512, 1001), (700, 256, 264)])
@pytest.mark.parametrize("gap", [0, 5, 48])
def test_nothing_beside_a_checkpoints_rows(rows, k, n, gap):
    """The C call with rows of its own: what lies between them, and the bytes behind the last block's, stay as they are."""
    x, w = randn(17, (rows, k), 1.0), randn(18, (n, k), 0.1)
    nb, row = -(-n // 16), n + gap
    data = torch.full((rows + 1, row), 99, device="cuda", dtype=torch.int8)
    scale = torch.full((rows + 1, nb + 3), 7, device="cuda", dtype=torch.uint8)
    y = torch.empty(rows, n, device="cuda", dtype=BF16)
    a = L.lipz_linear_checkpoint_args()
    a.struct_size, a.call.struct_size = L.ctypes.sizeof(a), L.ctypes.sizeof(a.call)
    a.call.groups, a.call.rows, a.call.k, a.call.n = 1, rows, k, n
    a.call.x, a.call.w = L.lipz_mat(x.data_ptr(), 0, k, L.LIPZ_BF16, 0), L.lipz_mat(w.data_ptr(), 0, k, L.LIPZ_BF16, 0)
    a.call.y = L.lipz_mat(y.data_ptr(), 0, n, L.LIPZ_BF16, 0)
    a.pre = L.lipz_blocks(data.data_ptr(), 0, row, scale.data_ptr(), 0, nb + 3)
    need = L.lipz_linear_checkpoint_workspace(a)
    space = torch.empty(need + 256, device="cuda", dtype=torch.uint8)
    a.call.workspace, a.call.workspace_bytes = (space.data_ptr() + 255) // 256 * 256, need
    L.lipz_linear_checkpoint(a, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    ref = ops.linear(x, w, keep="int8")
    assert torch.equal(y, ref[0])
    assert torch.equal(data[:rows, :n], ref[1].data) and torch.equal(scale[:rows, :nb], ref[1].scale)
    assert (data[:rows, n:] == 99).all() and (data[rows] == 99).all()
    assert (scale[:rows, nb:] == 7).all() and (scale[rows] == 7).all()


BACKWARDS = [(1, 1, 64, 32), (1, 37, 500, 1000), (1, 777, 500, 1001), (3, 100, 256, 512), (2, 65, 513, 77),
             (1, 1500, 784, 264), (1, 3000, 40, 24), (1, 0, 64, 32), (1, 9, 17, 1)]


@pytest.mark.parametrize("groups,rows,k,n", BACKWARDS)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("whole", [True, False])
def test_linear_backward_over_checkpoints(groups, rows, k, n, act, whole):
    """The bits of the same call over the bf16 values, whatever of x and pre is a checkpoint."""
    shape = (lambda *s: norm_shape(groups, *s))
    x, w = ops.checkpoint_rows(randn(21, shape(rows, k), 1.0)), randn(22, shape(n, k), k ** -0.5)
    pre, dy = ops.checkpoint_rows(randn(23, shape(rows, n), 1.0)), randn(24, shape(rows, n), 0.1)
    if not whole:  # rows at any byte
        x, pre = (ops.Checkpoint(c.data.contiguous(), c.scale) for c in (x, pre))
    xv, prev = ops.restore_rows(x), ops.restore_rows(pre)
    ref = ops.linear_backward(dy, xv, w, act=act, slope=SLOPE, pre=prev if act != "none" else None)
    for xx, pp in ((x, pre), (xv, pre), (x, prev)):
        got = ops.linear_backward(dy, xx, w, act=act, slope=SLOPE, pre=pp if act != "none" else None)
        for a, b, name in zip(got, ref, ("dx", "dw", "db")):
            assert torch.equal(a, b), name
    for wants in (dict(want_dx=False), dict(want_dw=False), dict(want_dx=False, want_dw=False),
                  dict(want_db=False, dw_dtype=F32)):
        got = ops.linear_backward(dy, x, w, act=act, slope=SLOPE, pre=pre if act != "none" else None, **wants)
        want = ops.linear_backward(dy, xv, w, act=act, slope=SLOPE, pre=prev if act != "none" else None, **wants)
        for a, b in zip(got, want):
            assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("groups,rows,k,n", [(1, 2100, 2056, 1992), (1, 300, 4104, 1000), (9, 270, 712, 360)])
def test_gradients_in_rows_16_bytes_off(groups, rows, k, n, dtype):
    """Widths of odd eights, whose rows begin on 16 bytes and on 32 by turns: against the formula in 64 bits over the
    values of the checkpoints (the errors of test_gpu_operators.py's test_linear_backward)."""
    shape = (lambda *s: norm_shape(groups, *s))
    x, w = ops.checkpoint_rows(randn(61, shape(rows, k))), randn(62, shape(n, k), k ** -0.5)
    pre, dy = ops.checkpoint_rows(randn(63, shape(rows, n), 1.5)), randn(64, shape(rows, n), 0.1)
    dx, dw, _ = ops.linear_backward(dy, x, w, act="silu", pre=pre, dx_dtype=dtype, dw_dtype=dtype)
    xv = ops.restore_rows(x)
    _, rx, rw, _ = backward_ref(dy, xv, w, "silu", ops.restore_rows(pre))
    size, delta, half = 1.2 * d(dy).abs(), 2.0 ** -8 + 2.0 ** -17, 2.0 ** -8 if dtype is BF16 else 2.0 ** -24
    within(dx, rx, half * rx.abs() + (delta + sum_error(n)) * (size @ d(w).abs()) + 1e-30, "dx")
    within(dw, rw, half * rw.abs() + (delta + sum_error(rows)) * (size.transpose(-1, -2) @ d(xv).abs()) + 1e-30, "dw")


@pytest.mark.parametrize("act", ACTS)
def test_slopes_at_the_ends(act):
    """Pre-activations from nothing to the largest: the bits of the same call over the bf16 values."""
    exps = torch.arange(-126, 122, device="cuda", dtype=F32)
    u = torch.cat([torch.exp2(exps) * s * 1.5 for s in (1, -1)] + [torch.linspace(-100, 100, 1008, device="cuda")])
    pre = ops.checkpoint_rows(u.reshape(-1, 1).expand(-1, 16).contiguous())
    dy, x, w = randn(28, (u.numel(), 16), 1.0), randn(29, (u.numel(), 8)), randn(30, (16, 8))
    ref = ops.linear_backward(dy, x, w, act=act, slope=SLOPE, pre=ops.restore_rows(pre) if act != "none" else None)
    got = ops.linear_backward(dy, x, w, act=act, slope=SLOPE, pre=pre if act != "none" else None)
    for a, b in zip(got, ref):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0))


def test_linear_backward_over_a_shared_checkpoint():
    """x that the groups share, and one whose scales alone they share."""
    groups, rows, k, n = 3, 50, 70, 90
    c = ops.checkpoint_rows(randn(25, (groups, rows, k), 1.0))
    w, dy = randn(26, (groups, n, k), 0.1), randn(27, (groups, rows, n), 0.1)
    for x in (ops.Checkpoint(c.data[:1].expand(groups, rows, k), c.scale[:1].expand(groups, rows, 5)),
              ops.Checkpoint(c.data, c.scale[:1].expand(groups, rows, 5)),
              ops.Checkpoint(c.data[:1].expand(groups, rows, k), c.scale)):
        for a, b in zip(ops.linear_backward(dy, x, w), ops.linear_backward(dy, ops.restore_rows(x), w)):
            assert torch.equal(a, b)


def test_refusals():
    x = randn(31, (8, 64))
    c = ops.checkpoint_rows(x)
    w, dy = randn(32, (32, 64)), randn(33, (8, 32))
    pre = ops.checkpoint_rows(dy)
    half = ops.Checkpoint(c.data, c.scale[:, :3])
    bad = [
        (lambda: ops.checkpoint_rows(x.half()), "dtype"),
        (lambda: ops.checkpoint_rows(x.t()), "adjacent"),
        (lambda: ops.checkpoint_rows(x.cpu()), "CUDA"),
        (lambda: ops.checkpoint_rows(x[0]), "rows, columns"),
        (lambda: ops.restore_rows(x), "checkpoint"),
        (lambda: ops.restore_rows(half), "scale has shape"),
        (lambda: ops.restore_rows(ops.Checkpoint(c.data.to(torch.uint8), c.scale)), "int8"),
        (lambda: ops.restore_rows(ops.Checkpoint(c.data, c.scale.to(torch.int8))), "int8"),
        (lambda: ops.restore_rows(ops.Checkpoint(c.data, c.scale.cpu())), "CUDA"),
        (lambda: ops.restore_rows(c, act="selu"), "act must"),
        (lambda: ops.restore_rows(c, out_dtype=torch.float16), "out_dtype"),
        (lambda: ops.linear(x, w, keep="int4"), "keep"),
        (lambda: ops.linear_backward(dy, half, w), "scale has shape"),
        (lambda: ops.linear_backward(dy, c, w, act="gelu"), "needs pre"),
        (lambda: ops.linear_backward(dy, c, w, act="gelu", pre=c), "pre has shape"),
        (lambda: ops.linear_backward(dy, c, w[:, :63], act="gelu", pre=pre), "w has shape"),
    ]
    for f, what in bad:
        with pytest.raises(L.LipzError) as e:
            f()
        assert e.value.code == L.LIPZ_ERR_INVALID and what in str(e.value), (what, str(e.value))
