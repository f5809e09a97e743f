"""The residual-block operators at the ends of their types' ranges: finite inputs whose results are finite by
the formulas give them."""

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
