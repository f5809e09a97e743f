"""Outputs over inputs are refused; outputs beside inputs in one buffer, and in the places that the calls allow,
are taken."""

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


@pytest.mark.parametrize("rows", [1, 3, 40, 600])
def test_an_output_over_an_input_is_refused(rows):
    buf, w, g = randn(rows + 1, 64), randn(64, 64), torch.ones(64, device="cuda")
    x, below = buf[:rows], buf[1:]
    before = buf.clone()
    calls = [lambda: ops.linear(x, w, out=x), lambda: ops.linear(x, w, residual=x, out=x)]
    if rows > 1:
        calls += [lambda: ops.linear(x, w, out=below),
                  lambda: ops.rmsnorm(x, g, residual=randn(rows, 64), sum_out=below)]
    for call in calls:
        with pytest.raises(L.LipzError, match="overlaps") as e:
            call()
        assert e.value.code == L.LIPZ_ERR_INVALID
    torch.cuda.synchronize()
    assert torch.equal(buf, before)


@pytest.mark.parametrize("groups,rows,k,n", [(1, 1, 64, 64), (1, 3, 200, 77), (1, 600, 256, 320), (4, 50, 96, 40)])
def test_outputs_beside_inputs_in_one_buffer(groups, rows, k, n):
    """Columns of one buffer, and groups woven row by row in it."""
    buf = randn(rows, groups, k + n).permute(1, 0, 2)
    w = randn(groups, n, k)
    x, out = buf[..., :k], buf[..., k:]
    want, _ = ops.linear(x.contiguous(), w, act="silu")
    got, _ = ops.linear(x, w, act="silu", out=out)
    assert got is out and torch.equal(out, want)
    both = randn(groups, rows, 2, k)
    a, b, g = both[:, :, 0], both[:, :, 1], torch.ones(groups, k, device="cuda")
    want = ops.rmsnorm(a.contiguous(), g, residual=b.contiguous())
    got = ops.rmsnorm(a, g, residual=b, sum_out=b)
    assert torch.equal(got.sum, want.sum) and torch.equal(got.y, want.y)


@pytest.mark.parametrize("rows", [3, 700])
def test_the_places_that_calls_allow(rows):
    x, res, w, g = randn(rows, 96), randn(rows, 96), randn(96, 96), torch.ones(96, device="cuda")
    want = ops.rmsnorm(x, g, residual=res)
    y, _ = ops.linear(x, w, residual=res)
    a, b = x.clone(), res.clone()
    got = ops.rmsnorm(a, g, residual=b, sum_out=a)
    assert got.sum is a and torch.equal(a, want.sum) and torch.equal(got.y, want.y)
    assert torch.equal(ops.linear(x, w, residual=b, out=b)[0], y) and torch.equal(b, y)
