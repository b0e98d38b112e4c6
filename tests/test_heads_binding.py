"""The binding of a head's operators: what it accepts (no GPU)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    from paper_2003_04296_gb300 import minw
    return minw


@pytest.mark.parametrize("limit", [1, 1.0, np.float32(1), np.float64(1), np.int64(1), torch.tensor(1.0)])
def test_one_limit_for_all_is_any_number(M, limit):
    assert len(M.TensorList([], limits=limit)) == 0


@pytest.mark.parametrize("limits", [[], (), np.zeros(0, dtype=np.float32), torch.zeros(0)])
def test_a_limit_for_each_is_any_sequence(M, limits):
    assert len(M.TensorList([], limits=limits)) == 0
    with pytest.raises(ValueError, match="limit per tensor"):
        M.TensorList([], limits=list(limits) + [1.0])
