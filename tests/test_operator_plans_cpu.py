"""How calls divide their work, as far as the workspace that they ask for shows it. No GPU is needed: without one the
library takes a device of 152 SMs."""

import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_1811_12843_gb300 import _build
    _build.build()
    import paper_1811_12843_gb300 as lib
    lib.load()
    return lib


@pytest.mark.parametrize("groups,rows,dim,parts", [
    (144, 100, 256, 1), (60, 100, 256, 1), (40, 300, 256, 1), (40, 6000, 256, 3), (60, 2000, 256, 2),
    (76, 6000, 64, 2), (90, 6000, 256, 1), (90, 1000, 1024, 3), (144, 1000, 1024, 1), (90, 100, 1024, 1),
    (20, 6000, 256, 7), (1, 8, 64, 1)])
def test_norm_backward_of_short_rows_fills_the_device(L, groups, rows, dim, parts):
    """Few turns, or no free SMs: one block per group, whose sums need no workspace."""
    def mat(at):
        return L.lipz_mat(at, rows * dim, dim, L.LIPZ_BF16, 0)

    a = L.lipz_rmsnorm_backward_args()
    a.struct_size = ctypes.sizeof(a)
    a.groups, a.rows, a.dim = groups, rows, dim
    a.dy, a.s, a.dx = mat(1 << 30), mat(2 << 30), mat(3 << 30)
    a.weight, a.rstd, a.dweight = (L.lipz_vec(i << 40, n) for i, n in ((1, dim), (2, rows), (3, dim)))
    assert L.lipz_rmsnorm_backward_workspace(a) == (groups * parts * dim * 4 if parts > 1 else 0)
