"""Host-side refusals of the calls on low-rank adapters: bad arguments return
their status before any device call, empty calls succeed, and the binding
rejects tensors of the wrong shape or type (no GPU)."""
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


COMMON = [
    dict(T=-1), dict(K=0), dict(O=0), dict(n=0), dict(r=0), dict(ldx=99), dict(x=None), dict(ids=None), dict(down=None),
    dict(up=None), dict(xt=2), dict(pt=-1), dict(x=P(FAKE + 2)), dict(x=P(FAKE + 1), xt=1), dict(down=P(FAKE + 2)),
    dict(up=P(FAKE + 1), pt=1), dict(ids=P(FAKE + 2)), dict(alpha=P(FAKE + 1)), dict(ws=None), dict(ws=P(FAKE + 8)), dict(wb=8)]
BIG = [dict(r=257), dict(n=1 << 24), dict(T=1 << 27), dict(K=(1 << 28) + 1, ldx=1 << 29), dict(n=(1 << 24) - 1, K=1 << 20, ldx=1 << 20)]


def _forward(M, **kw):
    a = dict(x=P(FAKE), xt=0, ldx=100, T=5, K=100, ids=P(FAKE), down=P(FAKE), up=P(FAKE), pt=0, n=3, r=4, alpha=None, base=None,
             bt=0, ldb=0, O=8, scale=None, shift=None, act=0, y=P(2 * FAKE), yt=0, ldy=8, h=None, ws=P(FAKE), wb=1 << 40)
    a.update(kw)
    return M.lib().minw_adapters(*a.values(), None)


@pytest.mark.parametrize("bad", COMMON + [
    dict(y=None), dict(yt=3), dict(ldy=7), dict(act=4), dict(act=-1), dict(y=P(FAKE + 2)), dict(base=P(FAKE), ldb=7),
    dict(base=P(FAKE), ldb=8, bt=2), dict(base=P(FAKE + 2), ldb=8), dict(base=P(2 * FAKE), ldb=9),
    dict(base=P(2 * FAKE), ldb=8, bt=1), dict(y=P(FAKE)), dict(scale=P(FAKE + 2)), dict(shift=P(FAKE + 1)), dict(h=P(FAKE + 2))])
def test_forward_refusals(M, bad):
    assert _forward(M, **bad) == M.MINW_EINVAL


@pytest.mark.parametrize("big", BIG)
def test_sizes(M, big):
    assert _forward(M, **big) == M.MINW_EUNSUPPORTED
    assert _backward(M, **big) == M.MINW_EUNSUPPORTED
    assert _w4(M, **big) == M.MINW_EUNSUPPORTED
    a = dict(T=5, K=100, O=8, n=3, r=4)
    a.update({k: v for k, v in big.items() if k in a})
    assert M.minw_adapters_workspace_bytes(*a.values()) == 0


def test_workspace(M):
    for bad in [(-1, 4, 4, 1, 1), (1, 0, 4, 1, 1), (1, 4, 0, 1, 1), (1, 4, 4, 0, 1), (1, 4, 4, 1, 0)]:
        assert M.minw_adapters_workspace_bytes(*bad) == 0
    need = M.minw_adapters_workspace_bytes(500, 100, 8, 3, 4)
    assert _forward(M, T=500, wb=need - 1) == M.MINW_EINVAL
    need = M.minw_adapters_workspace_bytes(500, 100, 8, 3, 4, True)
    assert _backward(M, T=500, wb=need - 1) == M.MINW_EINVAL


def test_no_rows(M):
    assert _forward(M, T=0, x=None, ids=None, y=None, ws=None, wb=0) == M.MINW_OK
    assert _w4(M, T=0, x=None, ids=None, y=None, ws=None, wb=0) == M.MINW_OK
    assert _backward(M, T=0, x=None, ids=None, dy=None, h=None, ddown=None, dup=None, ws=None, wb=0) == M.MINW_OK
    assert _backward(M, dx=None, ddown=None, dup=None, ws=None, wb=0) == M.MINW_OK


def _w4(M, **kw):
    a = dict(x=P(FAKE), xt=0, ldx=100, T=5, codes=P(FAKE), scales=P(FAKE), O=8, K=100, group=32, ids=P(FAKE), down=P(FAKE),
             up=P(FAKE), pt=0, n=3, r=4, alpha=None, scale=None, shift=None, act=0, y=P(2 * FAKE), yt=0, ldy=8, ws=P(FAKE),
             wb=1 << 40)
    a.update(kw)
    return M.lib().minw_w4_adapters(*a.values(), None)


@pytest.mark.parametrize("bad", COMMON + [
    dict(y=None), dict(yt=3), dict(ldy=7), dict(act=4), dict(y=P(FAKE)), dict(codes=None), dict(codes=P(FAKE + 8)), dict(scales=None),
    dict(group=48), dict(scales=P(FAKE + 1)), dict(scale=P(FAKE + 2)), dict(y=P(2 * FAKE + 2))])
def test_w4_refusals(M, bad):
    assert _w4(M, **bad) == M.MINW_EINVAL


def _backward(M, **kw):
    a = dict(x=P(FAKE), xt=0, ldx=100, T=5, K=100, ids=P(FAKE), down=P(FAKE), up=P(FAKE), pt=0, n=3, r=4, alpha=None, h=P(FAKE),
             dy=P(2 * FAKE), dt=0, ldd=8, O=8, dx=P(3 * FAKE), ldo=100, acc=0, ddown=P(4 * FAKE), dup=P(5 * FAKE), ws=P(FAKE),
             wb=1 << 40)
    a.update(dict(ldo=kw.get("ldx", 100)) if "K" in kw else {}, **kw)
    return M.lib().minw_adapters_backward(*a.values(), None)


@pytest.mark.parametrize("bad", COMMON + [
    dict(dy=None), dict(h=None), dict(dt=5), dict(ldd=7), dict(ldo=99), dict(dy=P(FAKE + 2)), dict(dx=P(FAKE + 2)),
    dict(dx=P(FAKE)), dict(dx=P(2 * FAKE)), dict(h=P(FAKE + 2)), dict(ddown=P(FAKE + 2)), dict(dup=P(FAKE + 1))])
def test_backward_refusals(M, bad):
    assert _backward(M, **bad) == M.MINW_EINVAL


def test_binding(M):
    torch = pytest.importorskip("torch")
    x, ids, down, up = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 3, 8), torch.zeros(2, 3, 5)
    with pytest.raises(ValueError):
        M.minw_adapters(x, ids, down, up, torch.zeros(3, 5))                   # rows
    with pytest.raises(ValueError):
        M.minw_adapters(x, ids, down, up, torch.zeros(4, 5))                   # on the host
    with pytest.raises(ValueError):
        M.minw_adapters(x, ids, down, up, torch.zeros(4, 5), base=torch.zeros(4, 6))
    with pytest.raises(ValueError):
        M.minw_adapters_backward(x, ids, down, up, None, torch.zeros(4, 5), dx=torch.zeros(4, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        M._pools(down, torch.zeros(2, 4, 5), 8, 5)
    with pytest.raises(ValueError):
        M._pools(down, up.bfloat16(), 8, 5)
    with pytest.raises(ValueError):
        M._ids(ids.long(), 4)
    with pytest.raises(ValueError):
        M._ids(ids, 5)
