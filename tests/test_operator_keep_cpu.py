"""What ``keep`` may be, without a GPU: it is looked at before the tensors are."""

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def L():
    from paper_1811_12843_gb300 import _build
    _build.build()
    import paper_1811_12843_gb300 as lib
    lib.load()
    return lib


@pytest.mark.parametrize("word", ["int8", "int4", ""])
def test_a_norm_that_keeps_nothing_in_8_bits_refuses_a_word(L, word):
    from paper_1811_12843_gb300 import operators as ops
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(L.LipzError) as e:
        ops.rmsnorm(x, torch.ones(64), keep=word)
    assert e.value.code == L.LIPZ_ERR_INVALID and "keep must be False or True" in str(e.value)


@pytest.mark.parametrize("keep", [False, True, 0, 1, None])
def test_truth_values_are_taken(L, keep):
    """(What is refused then are tensors that are not on a GPU.)"""
    from paper_1811_12843_gb300 import operators as ops
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(L.LipzError) as e:
        ops.rmsnorm(x, torch.ones(64), keep=keep)
    assert "CUDA" in str(e.value)
