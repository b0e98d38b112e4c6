"""Host-side refusals of the calls on lists of matrices: bad arguments return
their status before any device call, empty lists succeed, and the binding
rejects what is no matrix (no GPU)."""
import ctypes
import math

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


def _list(M, *entries):
    arr = (M.Matrix * max(1, len(entries)))()
    for e, kw in zip(arr, entries):
        a = dict(data=FAKE, ld=20, rows=10, cols=20, type=0, limit=1.0)
        a.update(kw)
        for k, v in a.items():
            setattr(e, k, v)
    return arr


def _orth(M, g=None, o=None, n=1, steps=5, ws=P(FAKE), wb=1 << 40):
    g = _list(M, dict()) if g is None else g
    o = _list(M, dict(data=1 << 20)) if o is None else o
    return M.lib().minw_orthogonalize(g, o, n, steps, ws, wb, None)


BAD = [dict(rows=-1), dict(cols=-1), dict(data=None), dict(ld=19), dict(type=2), dict(type=-1), dict(data=FAKE + 2),
       dict(data=FAKE + 1, type=1)]


@pytest.mark.parametrize("bad", BAD)
def test_matrices(M, bad):
    assert _orth(M, g=_list(M, bad)) == M.MINW_EINVAL
    assert _orth(M, o=_list(M, bad)) == M.MINW_EINVAL
    assert _orth(M, g=_list(M, {}, bad), o=_list(M, dict(data=1 << 20), dict(data=1 << 21)), n=2) == M.MINW_EINVAL
    assert M.lib().minw_orthogonal_workspace_bytes(_list(M, bad), 1) == 0


def test_lists(M):
    E = M.MINW_EINVAL
    g, o = _list(M, {}), _list(M, dict(data=1 << 20))
    need = M.lib().minw_orthogonal_workspace_bytes(g, 1)
    assert need > 0
    assert _orth(M, n=-1) == E
    assert M.lib().minw_orthogonalize(None, o, 1, 5, P(FAKE), need, None) == E
    assert M.lib().minw_orthogonalize(g, None, 1, 5, P(FAKE), need, None) == E
    for steps in (0, -1, 11):
        assert _orth(M, steps=steps) == E
    assert _orth(M, ws=None) == E and _orth(M, ws=P(FAKE + 8)) == E and _orth(M, wb=need - 1) == E
    for other in (dict(rows=9), dict(cols=19), dict(rows=20, cols=10)):
        assert _orth(M, o=_list(M, dict(data=1 << 20, **other))) == E
    # in place with another type or row length
    assert _orth(M, o=_list(M, dict(type=1))) == E and _orth(M, o=_list(M, dict(ld=24))) == E
    assert _orth(M, n=0, g=_list(M), o=_list(M), ws=None, wb=0) == M.MINW_OK
    assert M.lib().minw_orthogonalize(None, None, 0, 5, None, 0, None) == M.MINW_OK
    empty = _list(M, dict(rows=0, data=None))
    assert _orth(M, g=empty, o=empty, ws=None, wb=0) == M.MINW_OK
    assert M.lib().minw_orthogonal_workspace_bytes(_list(M), -1) == 0
    assert M.lib().minw_orthogonal_workspace_bytes(None, 1) == 0


def test_sizes(M):
    for big in (dict(rows=(1 << 22) + 1), dict(rows=1 << 16, cols=1 << 16, ld=1 << 16)):
        assert _orth(M, g=_list(M, big), o=_list(M, dict(big, data=1 << 20))) == M.MINW_EUNSUPPORTED
        assert M.lib().minw_orthogonal_workspace_bytes(_list(M, big), 1) == 0


def test_workspace_grows_with_the_list(M):
    one = M.lib().minw_orthogonal_workspace_bytes(_list(M, {}), 1)
    two = M.lib().minw_orthogonal_workspace_bytes(_list(M, {}, dict(rows=1000, cols=1000, ld=1000)), 2)
    assert 0 < one < two


@pytest.mark.parametrize("kw", [dict(lr=math.nan), dict(lr=math.inf), dict(mu=math.nan), dict(mu=math.inf),
                                dict(w=[dict(limit=-1.0)]), dict(w=[dict(limit=math.nan)]), dict(w=None),
                                dict(m=[dict(data=1 << 21, type=1)]), dict(m=[dict(data=None)]), dict(m=[dict(data=FAKE)]),
                                dict(m=[dict(data=1 << 20)]), dict(w=[dict(data=FAKE)]), dict(steps=0), dict(n=-1)])
def test_update(M, kw):
    a = dict(w=[{}], m=[dict(data=1 << 21)], lr=0.1, mu=0.9, steps=5, n=1)
    a.update(kw)
    w = a["w"] and _list(M, *(dict(dict(data=1 << 20), **e) for e in a["w"]))
    m = a["m"] and _list(M, *a["m"])
    assert M.lib().minw_sgd_orthogonal(w, m, _list(M, {}), a["n"], a["steps"], a["mu"], 1, a["lr"], P(FAKE), 1 << 40,
                                       None) == M.MINW_EINVAL


def test_binding(M):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        M.MatrixList([torch.zeros(4)])                        # a vector
    with pytest.raises(ValueError):
        M.MatrixList([torch.zeros(4, 4)])                     # on the host
    with pytest.raises(ValueError):
        M.MatrixList([], limits=[1.0])
