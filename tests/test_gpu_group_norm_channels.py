"""The group norm with groups of one channel (an instance norm) in wide vectors,
both directions, against its formula in 64 bits (bounds: test_gpu_group_norm)."""
import pytest

pytest.importorskip("torch")

from tests.test_gpu_group_norm import M, test_backward as backward, test_forward as forward  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [8, 64, 256, 1024])
@pytest.mark.parametrize("types", ["bb", "bf", "fb", "ff"])
@pytest.mark.parametrize("B,P,act", [(2, 64, 0), (3, 129, 3)])
def test_groups_of_one_channel(M, B, P, C, types, act):  # noqa: F811
    case = (B, P, C, C, C, 0, types[0], types[1], act)
    forward(M, case)
    backward(M, case)
