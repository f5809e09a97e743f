"""Checkpoints whose rows lie past 2^31 elements, in the products that keep and read them: a block of rows over and over,
so that each copy has the bits of the first."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_1811_12843_gb300 import operators as ops
    from test_gpu_operators import d, randn, sum_error, within

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def same_copies(t, rows):
    """Every block of rows has the first one's bits."""
    t = t.view(-1, rows, t.shape[-1])
    return all(torch.equal(t[i], t[0]) for i in range(1, t.shape[0], 97)) and torch.equal(t[-1], t[0])


@pytest.mark.parametrize("n", [256, 250])
def test_products_over_rows_past_two_gigaelements(n):
    """(250 columns: rows of bytes that lie 256 apart, and off the 16-byte grid in bf16.)"""
    rows, copies, k = 4096, 2080, 256
    block, w, b = randn(1, (rows, k), 1.0), randn(2, (n, k), k ** -0.5), randn(3, (n,), 0.3, F32)
    x = block.repeat(copies, 1)
    y, pre = ops.linear(x, w, b, act="silu", keep="int8")
    assert pre.data.stride(0) * x.shape[0] > 2 ** 31 and x.numel() > 2 ** 31
    u = d(block) @ d(w).T + d(b)
    err = sum_error(k) * (d(block).abs() @ d(w).abs().T + d(b).abs())
    first = ops.Checkpoint(pre.data[:rows], pre.scale[:rows])
    unit = torch.exp2(d(first.scale) - 127).repeat_interleave(16, dim=-1)[:, :n]
    within(ops.restore_rows(first), u, unit / 2 + err, "pre")
    assert same_copies(y, rows) and same_copies(pre.scale, rows)
    assert same_copies(pre.data.as_strided((x.shape[0], n), pre.data.stride()).contiguous(), rows)
    xc = ops.checkpoint_rows(x)
    assert same_copies(xc.data, rows) and same_copies(xc.scale, rows)
    del x
    dy = y
    dx, dw, db = ops.linear_backward(dy, xc, w, act="silu", pre=pre, dw_dtype=F32)
    assert same_copies(dx, rows)
    one = ops.linear_backward(dy[:rows], ops.Checkpoint(xc.data[:rows], xc.scale[:rows]), w, act="silu", pre=first,
                              dw_dtype=F32)
    # (sums of `copies` times the terms, by chains of as many additions at most as a sum of all rows has: sum_error; the
    # first block's own are off by that of its rows)
    s, p = torch.sigmoid(d(ops.restore_rows(first))), d(ops.restore_rows(first))
    du = (d(dy[:rows]) * s * (1 + p * (1 - s))).abs() * (1 + 2.0 ** -7)
    size = du.T @ d(ops.restore_rows(ops.Checkpoint(xc.data[:rows], xc.scale[:rows]))).abs()
    lost = sum_error(rows * copies) + sum_error(rows)
    within(dw / copies, d(one[1]), lost * size + 1e-30, "dw")
    within(db / copies, d(one[2]), lost * du.sum(dim=0) + 1e-30, "db")
