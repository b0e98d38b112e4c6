"""The vectors beside a head's tensors (gamma, beta, statistics, scales, shifts,
parameter gradients): off the boundary of an fp32 value they are refused on the
host, where a kernel's load would fault (no GPU: every call ends before a launch)."""
import ctypes

import pytest

P = ctypes.c_void_p
FAKE = 4096                               # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    from paper_2003_04296_gb300 import minw
    minw.lib()
    return minw


@pytest.fixture(autouse=True)
def no_gpu():
    """A call that these checks let through would be launched on addresses that hold nothing."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("runs on a machine without a GPU")


OFF = [FAKE + 1, FAKE + 2, FAKE + 3, FAKE + 6]


@pytest.mark.parametrize("at", OFF)
@pytest.mark.parametrize("which", range(4))
def test_group_norm(M, which, at):
    v = [P(FAKE)] * 4
    v[which] = P(at)
    gamma, beta, mean, rstd = v
    assert M.lib().minw_group_norm(P(FAKE), 0, 64, gamma, beta, 2, 9, 64, 8, 1e-5, 0, P(2 * FAKE), 0, 64, mean, rstd,
                                   P(FAKE), 1 << 30, None) == M.MINW_EINVAL


@pytest.mark.parametrize("at", OFF)
@pytest.mark.parametrize("which", range(6))
@pytest.mark.parametrize("B", [0, 2])
def test_group_norm_backward(M, which, at, B):
    v = [P(FAKE)] * 6
    v[which] = P(at)
    gamma, beta, mean, rstd, dgamma, dbeta = v
    assert M.lib().minw_group_norm_backward(P(FAKE), 0, 64, P(2 * FAKE), 0, 64, gamma, beta, mean, rstd, B, 9, 64, 8, 0,
                                            P(3 * FAKE), 64, dgamma, dbeta, P(FAKE), 1 << 30, None) == M.MINW_EINVAL


@pytest.mark.parametrize("at", OFF)
def test_pack(M, at):
    q = M.quant(2, (0.5, 0.0, 0.0))
    assert M.lib().minw_pack_w4(P(FAKE), 0, 4, 100, 32, ctypes.byref(q), P(at), P(FAKE), P(FAKE), None) == M.MINW_EINVAL


@pytest.mark.parametrize("at", OFF)
@pytest.mark.parametrize("which", range(2))
def test_matvec(M, which, at):
    v = [P(FAKE)] * 2
    v[which] = P(at)
    assert M.lib().minw_w4_matvec(P(FAKE), 1, 100, 1, P(FAKE), P(FAKE), 8, 100, 32, v[0], v[1], 0, P(FAKE), 0, 8,
                                  None) == M.MINW_EINVAL
