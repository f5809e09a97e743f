"""What the documentation says of how far results may be off, where that is reached."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_1811_12843_gb300 import operators as ops
    from test_gpu_operators import d, norm_shape, randn, within

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_an_element_of_a_checkpoint_is_off_by_127_5_ths_at_most(dtype):
    """A block whose largest is 127.5 has multiples of 2: 1 lies in the middle of two of them, and 2^-7 of 127.5 is less."""
    x = randn(1, (64, 160), 1.0, dtype)
    x[0], x[0, ::16] = 1.0, 127.5
    off = (d(ops.restore_rows(ops.checkpoint_rows(x))) - d(x)).abs().unflatten(-1, (-1, 16)).amax(dim=-1)
    top = d(x).abs().unflatten(-1, (-1, 16)).amax(dim=-1)
    assert (off <= top / 127.5).all() and (off[0] == 1.0).all() and (off[0] > 2.0 ** -7 * top[0]).all()
