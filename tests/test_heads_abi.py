"""Host-side refusals of the head's entry points (group norm, clipped updates,
4-bit products): bad arguments return their status before any device call,
empty calls succeed, and the binding rejects tensors of the wrong shape, type
or strides (no GPU)."""
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


def _norm(M, **kw):
    a = dict(x=P(FAKE), xt=0, ldx=64, gamma=None, beta=None, B=2, Pn=9, C=64, G=8, eps=1e-5, act=0, y=P(2 * FAKE),
             yt=0, ldy=64, mean=None, rstd=None, ws=P(FAKE), wb=1 << 30)
    a.update(kw)
    return M.lib().minw_group_norm(a["x"], a["xt"], a["ldx"], a["gamma"], a["beta"], a["B"], a["Pn"], a["C"], a["G"],
                                   a["eps"], a["act"], a["y"], a["yt"], a["ldy"], a["mean"], a["rstd"], a["ws"],
                                   a["wb"], None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(B=-1), dict(Pn=0), dict(C=0), dict(G=0), dict(G=7), dict(ldx=63), dict(ldy=63),
    dict(xt=2), dict(yt=-1), dict(act=4), dict(act=-1), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(x=P(FAKE + 2)), dict(y=P(FAKE + 1), yt=1), dict(ws=None), dict(ws=P(FAKE + 8)),
    dict(wb=16), dict(y=P(FAKE), yt=1), dict(y=P(FAKE), ldy=72)])
def test_group_norm_refusals(M, bad):
    need = M.minw_group_norm_workspace_bytes(2, 9, 64, 8)
    if {"ws", "wb"} & set(bad) and need == 0:
        pytest.skip("no workspace for this shape")
    assert _norm(M, **bad) == M.MINW_EINVAL


def test_group_norm_sizes(M):
    assert _norm(M, Pn=1 << 30) == M.MINW_EUNSUPPORTED
    assert _norm(M, B=0, x=None, y=None, ws=None, wb=0) == M.MINW_OK
    for bad in [(0, 4, 8, 2), (1, 0, 8, 2), (1, 4, 8, 3), (1, 1 << 30, 8, 2), (-1, 4, 8, 2)]:
        assert M.minw_group_norm_workspace_bytes(*bad) == 0
        assert M.minw_group_norm_workspace_bytes(*bad, True) == 0


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(B=-1), dict(Pn=0), dict(G=5),
    dict(ldx=63), dict(lddy=63), dict(lddx=63), dict(xt=3), dict(dt=3), dict(act=7), dict(dy=P(FAKE + 1)),
    dict(dx=P(FAKE + 3)), dict(dx=P(FAKE), lddx=65), dict(dt=1, dx=P(3 * FAKE), dy=P(3 * FAKE)), dict(ws=None),
    dict(wb=0), dict(ws=P(FAKE + 4))])
def test_group_norm_backward_refusals(M, bad):
    a = dict(x=P(FAKE), xt=0, ldx=64, dy=P(2 * FAKE), dt=0, lddy=64, mean=P(FAKE), rstd=P(FAKE), B=2, Pn=9, C=64, G=8,
             act=0, dx=P(3 * FAKE), lddx=64, ws=P(FAKE), wb=1 << 30)
    a.update(bad)
    assert M.lib().minw_group_norm_backward(a["x"], a["xt"], a["ldx"], a["dy"], a["dt"], a["lddy"], None, None,
                                            a["mean"], a["rstd"], a["B"], a["Pn"], a["C"], a["G"], a["act"], a["dx"],
                                            a["lddx"], None, None, a["ws"], a["wb"], None) == M.MINW_EINVAL


def _tensors(M, *entries):
    arr = (M.Tensor * max(1, len(entries)))()
    for e, (data, n, t, limit) in zip(arr, entries):
        e.data, e.n, e.type, e.limit = data, n, t, limit
    return arr


def test_gradient_list_refusals(M):
    L = M.lib()
    ok = _tensors(M, (FAKE, 10, 0, 1.0))
    ws, wb = P(FAKE), M.minw_grad_workspace_bytes(1)
    norm = P(FAKE)
    E = M.MINW_EINVAL
    assert L.minw_grad_norm(ok, -1, norm, ws, wb, None) == E
    assert L.minw_grad_norm(None, 1, norm, ws, wb, None) == E
    assert L.minw_grad_norm(ok, 1, None, ws, wb, None) == E
    assert L.minw_grad_norm(ok, 1, norm, None, wb, None) == E
    assert L.minw_grad_norm(ok, 1, norm, ws, wb - 1, None) == E
    assert L.minw_grad_norm(ok, 1, norm, P(FAKE + 8), wb, None) == E
    assert L.minw_grad_norm(ok, 1, P(FAKE + 2), ws, wb, None) == E
    for e in [(FAKE, -1, 0, 1.0), (None, 3, 0, 1.0), (FAKE, 3, 2, 1.0), (FAKE + 2, 3, 0, 1.0), (FAKE + 1, 3, 1, 1.0)]:
        assert L.minw_grad_norm(_tensors(M, e), 1, norm, ws, wb, None) == E, e
    assert L.minw_grad_norm(_tensors(M, (FAKE, 1 << 46, 0, 1.0)), 1, norm, ws, wb, None) == M.MINW_EUNSUPPORTED
    # clipping: lists that differ, a limit of the norm that is none
    for o in [(FAKE, 9, 0, 1.0), (FAKE, 10, 1, 1.0), (None, 10, 0, 1.0)]:
        assert L.minw_grad_clip(ok, _tensors(M, o), 1, 1.0, norm, ws, wb, None) == E, o
    assert L.minw_grad_clip(ok, None, 1, 1.0, norm, ws, wb, None) == E
    for m in (0.0, -1.0, float("nan"), float("inf")):
        assert L.minw_grad_clip(ok, ok, 1, m, norm, ws, wb, None) == E
        assert L.minw_sgd_clip_norm(ok, ok, 1, m, 0.1, norm, ws, wb, None) == E
    # the update: the learning rate, a weight's limit
    assert L.minw_sgd_clip_norm(ok, ok, 1, 1.0, float("nan"), norm, ws, wb, None) == E
    assert L.minw_sgd_clip_norm(_tensors(M, (FAKE, 10, 0, -1.0)), ok, 1, 1.0, 0.1, norm, ws, wb, None) == E
    assert L.minw_sgd_clip_norm(_tensors(M, (FAKE, 10, 0, float("nan"))), ok, 1, 1.0, 0.1, norm, ws, wb, None) == E
    assert M.minw_grad_workspace_bytes(-1) == 0
    assert 0 < M.minw_grad_workspace_bytes(0) <= M.minw_grad_workspace_bytes(1) < M.minw_grad_workspace_bytes(5000)


@pytest.mark.parametrize("bad", [
    dict(w=None), dict(codes=None), dict(scales=None), dict(O=0), dict(K=0), dict(group=0), dict(group=-32),
    dict(group=16), dict(group=48), dict(group=96), dict(group=192), dict(t=2), dict(w=P(FAKE + 2)),
    dict(codes=P(FAKE + 8)), dict(scales=P(FAKE + 1)), dict(bits=4)])
def test_pack_refusals(M, bad):
    a = dict(w=P(FAKE), t=0, O=4, K=100, group=32, codes=P(FAKE), scales=P(FAKE), bits=0)
    a.update(bad)
    q = ctypes.byref(M.quant(a["bits"])) if a["bits"] else None
    assert M.lib().minw_pack_w4(a["w"], a["t"], a["O"], a["K"], a["group"], q, None, a["codes"], a["scales"],
                                None) == M.MINW_EINVAL


def _matvec(M, **kw):
    a = dict(x=P(FAKE), xt=1, ldx=100, T=1, codes=P(FAKE), scales=P(FAKE), O=8, K=100, group=32, act=0, y=P(FAKE), yt=0,
             ldy=8)
    a.update(kw)
    return M.lib().minw_w4_matvec(a["x"], a["xt"], a["ldx"], a["T"], a["codes"], a["scales"], a["O"], a["K"],
                                  a["group"], None, None, a["act"], a["y"], a["yt"], a["ldy"], None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(codes=None), dict(scales=None), dict(y=None), dict(T=-1), dict(O=0), dict(K=0), dict(group=100),
    dict(ldx=99), dict(ldy=7), dict(xt=2), dict(yt=2), dict(act=9), dict(codes=P(FAKE + 4)), dict(x=P(FAKE + 1)),
    dict(y=P(FAKE + 2)), dict(scales=P(FAKE + 1))])
def test_matvec_refusals(M, bad):
    assert _matvec(M, **bad) == M.MINW_EINVAL


def test_matvec_of_no_vector(M):
    assert _matvec(M, T=0, x=None, y=None) == M.MINW_OK
    assert _matvec(M, K=(1 << 28) + 1, ldx=1 << 29) == M.MINW_EUNSUPPORTED


def test_w4_shapes(M):
    assert M.w4_shapes(5, 1, 32) == ((5, 64), (5, 1))
    assert M.w4_shapes(5, 128, 64) == ((5, 64), (5, 2))
    assert M.w4_shapes(5, 129, 128) == ((5, 128), (5, 2))


def test_binding_rejects_host_tensors_and_types(M):
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 8)
    with pytest.raises(ValueError):
        M.minw_group_norm(x, None, None, 2, 1e-5, x)
    with pytest.raises(ValueError):
        M.minw_group_norm(x, None, None, 2, 1e-5, torch.zeros(2, 4, 9))
    with pytest.raises(ValueError):
        M.TensorList([torch.zeros(3)])
    with pytest.raises(ValueError):
        M._value_type(torch.zeros(3, dtype=torch.float16))
    with pytest.raises(ValueError):
        M.minw_grad_clip(M.TensorList([]), [torch.zeros(1)], 1.0, None, None)
    with pytest.raises(ValueError):
        M.minw_w4_matvec(torch.zeros(2, 8), torch.zeros(3, 64, dtype=torch.uint8), torch.zeros(3, 1), 32,
                         torch.zeros(3, 3))
