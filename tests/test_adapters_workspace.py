"""Workspace of the calls on adapters: few rows need none that grows with the
number of adapters, and their terms beside 4-bit weights 4 bytes a value (no GPU)."""
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


@pytest.mark.parametrize("T", [1, 5, 32, 33, 64])
@pytest.mark.parametrize("O", [1, 10, 4096])
def test_few_rows(M, T, O):
    few, many = M.minw_adapters_workspace_bytes(T, 100, O, 3, 8), M.minw_adapters_workspace_bytes(T, 100, O, 1 << 20, 8)
    assert few == many == max(16, min(T, 32) * O * 4)
    assert M.minw_adapters_workspace_bytes(T, 100, O, 1 << 20, 8, True) > 1 << 20        # the backward sorts rows by user


def test_more_rows(M):
    at = [M.minw_adapters_workspace_bytes(T, 100, 50, 2000, 8) for T in (64, 65, 1000, 100000)]
    assert at == sorted(at) and at[1] > 2000 * 33 * 4                                    # counts of each user
    assert M.minw_adapters_workspace_bytes(0, 100, 50, 3, 8) == 16


def test_w4_takes_its_terms_alone(M):
    a = dict(x=P(FAKE), xt=0, ldx=100, T=1000, codes=P(FAKE), scales=P(FAKE), O=8, K=100, group=32, ids=P(FAKE), down=P(FAKE),
             up=P(FAKE), pt=0, n=3, r=4, alpha=None, scale=None, shift=None, act=0, y=P(2 * FAKE), yt=0, ldy=8, ws=P(FAKE),
             wb=32 * 8 * 4 - 1)
    assert M.lib().minw_w4_adapters(*a.values(), None) == M.MINW_EINVAL
    a.update(T=5, wb=5 * 8 * 4 - 1)
    assert M.lib().minw_w4_adapters(*a.values(), None) == M.MINW_EINVAL
