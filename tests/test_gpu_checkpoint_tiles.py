"""Products that keep a checkpoint, in the tiles that large ones take: 256 x 256 on pairs of CTAs, whose result warps hold
64 columns each in turns of 16, and 256 x 128. The tiles are those of a device of 152 SMs, and each case says which.

Elements are within half a step of their block and the error of a sum of k products. That bound is wide enough for sums
that lose far more than these do, so the multiples' mean square error has a limit of its own. A multiple turns where the
sum's error d carries it past the middle between two, with a probability of |d| / 2^e, and moves by 2^e: the mean square
is the mean of 2^e |d|. A sum in tensor memory truncates after each step of 16 bf16 (32 e4m3) of k: by something under
2^-23 of the sum so far, half of it on average, always towards zero. Over N steps of random sign, whose sum so far grows
with the root of their number, that comes to a standard deviation of up to 2^-24 N sqrt(1 / 3) of the sum's own (a mean
magnitude of 0.8 of it): 7.0e-6 for one sum over k = 4096 (N = 256), and half of that where the sum lies near the next
power of two. Sums of n_i chunks of four steps lose 2^-24 sqrt(sum of (4 n_i)^3 / (3 N)): 15, 15, 9, 9, 9 and 7 chunks
0.7e-6 to 1.3e-6. The limit is 1.5 2^-20 = 1.4e-6 of the values' root mean square: above what these sums lose, and below
one sum of 4096. (Error of the multiples, of their root mean square, at 8192 x 4096 -> 8192: 1.18e-4, limit 1.86e-4, one
sum 2.84e-4.) Products of e4m3 have fewer bits, of which a sum has to drop fewer: one sum over k of 7299 to 8192 is off
by 8.4e-5 to 9.0e-5, these by 4.1e-5 to 5.4e-5, and their limit, 0.875 2^-22, comes to 7.1e-5.
"""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import paper_1811_12843_gb300 as L
    from launched import kernels
    from paper_1811_12843_gb300 import operators as ops
    from test_gpu_checkpoints import blocks64, product
    from test_gpu_operators import act64, d, randn, sum_error, within

BF16, F32 = torch.bfloat16, torch.float32
LOST, LOST_E4M3 = 1.5 * 2.0 ** -20, 0.875 * 2.0 ** -22


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def in_tiles_of_256(names, e4m3=False):
    """256 x 256 on pairs, sums in registers."""
    return any("k_gemm_opILi%dELi2ELi256ELb1EfLb0ELb0ELb0ELi1EE" % (2 if e4m3 else 1) in n for n in names)


def in_pairs_of_128(names, e4m3, out_dtype):
    """256 x 128 on pairs, sums in registers; bf16 results by TMA or not."""
    return any("k_gemm_opILi%dELi2ELi128ELb1EfLb%dELb0ELb0ELi%dEE" % (2 if e4m3 else 1, via, 1 if out_dtype is BF16 else 2)
               in n for n in names for via in (0, 1))


def check_pre(pre, u, size, k, lost):
    """pre against the product in 64 bits: each element, each byte, and the multiples' error by and large."""
    err = sum_error(k) * size
    n = u.shape[-1]
    unit = torch.exp2(d(pre.scale) - 127).repeat_interleave(16, dim=-1)[..., :n]
    within(ops.restore_rows(pre), u, unit / 2 + err, "pre")
    byte = [blocks64(u.abs() + s * err)[1] for s in (1, 0)]
    low = blocks64((u.abs() - err).clamp(min=0))[1]
    got = pre.scale.to(torch.int64)
    assert ((got >= low) & (got <= byte[0])).all()
    ref = blocks64(u)[2]
    assert (got != byte[1]).double().mean() < 1e-4  # (err is 2^-8 of a block's largest at most; these are off by 2^-20)
    got = d(ops.restore_rows(pre))
    same = (pre.scale.to(torch.int64) == byte[1]).repeat_interleave(16, dim=-1)[..., :n]
    rms = ref.square().mean().sqrt()
    off = torch.where(same, got - ref, torch.zeros_like(ref)).square().mean()
    limit = unit.mean() * lost * rms
    assert off < limit, (float(off.sqrt() / rms), float(limit.sqrt() / rms))


# rows and columns that fill their last tiles in part; a checkpoint's rows of 95, 319, 128, 62, 303, 110 and 191 blocks
# (its bytes by words, by halves, one by one); rows that TMA does not take; columns left out of a block; groups
TILES = [(1, 8692, 4608, 1512, False, "none", False), (2, 1246, 4372, 5096, False, "none", False),
         (1, 6128, 7616, 2040, False, "silu", True), (7, 1769, 7314, 984, False, "silu", True),
         (7, 1017, 5343, 4841, False, "gelu", False), (1, 8192, 4096, 8192, False, "silu", False),
         (2, 3575, 7299, 1760, True, "none", False), (2, 3067, 7480, 3048, True, "none", True)]


@pytest.mark.parametrize("groups,rows,k,n,e4m3,act,res", TILES)
def test_tiles_of_256(groups, rows, k, n, e4m3, act, res):
    x, w, b, xs, ws, u, size = product(groups, rows, k, n, e4m3)
    residual = randn(14, u.shape, 1.0) if res else None

    def call():
        return ops.linear(x, w, b, act=act, residual=residual, x_scale=xs, w_scale=ws, keep="int8")

    assert in_tiles_of_256(kernels(call), e4m3)
    y, pre = call()
    check_pre(pre, u, size, k, LOST_E4M3 if e4m3 else LOST)
    ref = act64(act, u) + (d(residual) if res else 0)
    within(y, ref, 2.0 ** -8 * ref.abs() * (1 + 2.0 ** -7) + 1.13 * sum_error(k) * size * (1 + 2.0 ** -8) +
           2.0 ** -17 * act64(act, u).abs() * (1 + u.abs()), act)
    again = call()
    assert torch.equal(y, again[0]) and torch.equal(pre.data, again[1].data) and torch.equal(pre.scale, again[1].scale)


@pytest.mark.parametrize("rows,k,n,e4m3,out_dtype", [
    (2048, 4096, 2048, False, BF16), (2048, 4096, 2048, False, F32), (2040, 4090, 2001, False, BF16),
    (2048, 8192, 2048, True, BF16)])
def test_sums_in_tiles_of_128(rows, k, n, e4m3, out_dtype):
    x, w, b, xs, ws, u, size = product(1, rows, k, n, e4m3)

    def call():
        return ops.linear(x, w, b, x_scale=xs, w_scale=ws, out_dtype=out_dtype, keep="int8")

    assert in_pairs_of_128(kernels(call), e4m3, out_dtype)
    y, pre = call()
    check_pre(pre, u, size, k, LOST_E4M3 if e4m3 else LOST)
    half = torch.finfo(out_dtype).eps / 2
    within(y, u, half * u.abs() * (1 + 2.0 ** -7) + sum_error(k) * size * (1 + 2.0 ** -7), "y")
    again = call()
    assert torch.equal(y, again[0]) and torch.equal(pre.data, again[1].data) and torch.equal(pre.scale, again[1].scale)


@pytest.mark.parametrize("gap,blocks", [(0, 0), (8, 1), (24, 3), (5, 2)])
def test_nothing_beside_the_rows_of_tiles_of_256(gap, blocks):
    """The C call: rows 1512 bytes and a gap apart (boundaries of 8, 16, 32 and 1 byte), their bytes 95 and some apart."""
    rows, k, n = 8692, 4608, 1512
    x, w = randn(17, (rows, k), 1.0), randn(18, (n, k), k ** -0.5)
    nb, row = -(-n // 16), n + gap
    data = torch.full((rows + 1, row), 99, device="cuda", dtype=torch.int8)
    scale = torch.full((rows + 1, nb + blocks), 7, device="cuda", dtype=torch.uint8)
    y = torch.empty(rows, n, device="cuda", dtype=BF16)
    a = L.lipz_linear_checkpoint_args()
    a.struct_size, a.call.struct_size = L.ctypes.sizeof(a), L.ctypes.sizeof(a.call)
    a.call.groups, a.call.rows, a.call.k, a.call.n = 1, rows, k, n
    a.call.x, a.call.w = L.lipz_mat(x.data_ptr(), 0, k, L.LIPZ_BF16, 0), L.lipz_mat(w.data_ptr(), 0, k, L.LIPZ_BF16, 0)
    a.call.y = L.lipz_mat(y.data_ptr(), 0, n, L.LIPZ_BF16, 0)
    a.pre = L.lipz_blocks(data.data_ptr(), 0, row, scale.data_ptr(), 0, nb + blocks)
    need = L.lipz_linear_checkpoint_workspace(a)
    space = torch.empty(need + 256, device="cuda", dtype=torch.uint8)
    a.call.workspace, a.call.workspace_bytes = (space.data_ptr() + 255) // 256 * 256, need

    def call():
        L.lipz_linear_checkpoint(a, torch.cuda.current_stream().cuda_stream)

    assert in_tiles_of_256(kernels(call))
    torch.cuda.synchronize()
    ref = ops.linear(x, w, keep="int8")
    assert torch.equal(y, ref[0])
    assert torch.equal(data[:rows, :n], ref[1].data) and torch.equal(scale[:rows, :nb], ref[1].scale)
    assert (data[:rows, n:] == 99).all() and (data[rows] == 99).all()
    assert (scale[:rows, nb:] == 7).all() and (scale[rows] == 7).all()


def test_a_nan_and_an_infinity_in_tiles_of_256():
    """They stay in their rows, whose blocks are all byte 255 (a row of NaN, and one of infinities or NaN)."""
    rows, k, n = 8692, 4608, 1512
    x, w = randn(19, (rows, k), 1.0), randn(20, (n, k), k ** -0.5)
    x[300, 7], x[8691, 4607] = float("nan"), float("inf")
    call = lambda: ops.linear(x, w, keep="int8")  # noqa: E731
    assert in_tiles_of_256(kernels(call))
    bad = (call()[1].scale == 255).all(dim=-1).nonzero().flatten().tolist()
    assert bad == [300, 8691] and int((call()[1].scale == 255).any(dim=-1).sum()) == 2
