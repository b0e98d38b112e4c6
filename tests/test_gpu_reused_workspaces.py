"""One workspace for call after call, each with other rows, users, inputs or
matrices, nothing waiting between: the same bits as a call by itself on a
workspace of its own.  (Kernels that start before the one ahead of them is
done read what earlier ones left in the workspace, at the same addresses every time.)"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _scratch(nbytes, fill):
    return torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("xt,yt", [("f", "f"), ("b", "b"), ("f", "b")])
def test_backward_of_changing_users(M, xt, yt):
    dt = {"f": torch.float32, "b": torch.bfloat16}
    gen = torch.Generator(device="cuda").manual_seed(1)
    K, O, n, r = 264, 328, 7, 16
    down, up = _rand(gen, n, r, K) / 16, _rand(gen, n, r, O) / 4
    calls = []
    for k in range(24):
        T = 65 + 53 * (k % 5)
        ids = torch.randint(-1, n, (T,), generator=gen, device="cuda").to(torch.int32)
        if k % 3 == 0:
            ids = ids.sort().values.flip(0).contiguous()
        calls.append(dict(x=_rand(gen, T, K).to(dt[xt]), ids=ids, h=_rand(gen, T, r), dy=_rand(gen, T, O).to(dt[yt])))
    most = M.minw_adapters_workspace_bytes(65 + 53 * 4, K, O, n, r, True)

    def outputs(c):
        return dict(dx=torch.full_like(c["x"], 7), ddown=torch.full_like(down, 7), dup=torch.full_like(up, 7))

    def call(c, o, ws):
        M.minw_adapters_backward(c["x"], c["ids"], down, up, c["h"], c["dy"], ddown=o["ddown"], dup=o["dup"], dx=o["dx"],
                                 workspace=ws)

    want = []
    for c in calls:
        o = outputs(c)
        call(c, o, _scratch(most, 0))
        torch.cuda.synchronize()
        want.append(o)
    got = [outputs(c) for c in calls]
    ws = _scratch(most, 255)
    torch.cuda.synchronize()
    for c, o in zip(calls, got):
        call(c, o, ws)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("t,ld", [("f", 1000), ("f", 1003), ("b", 1000), ("b", 1003)])
def test_beside_4_bit_weights_on_inputs_that_change_in_place(M, t, ld):
    """x and the scales are written by a kernel right ahead of the call, at the same addresses."""
    dt = {"f": torch.float32, "b": torch.bfloat16}[t]
    gen = torch.Generator(device="cuda").manual_seed(2)
    T, K, O, n, r, group = 9, 1000, 200, 4, 8, 32
    w = _rand(gen, O, K) / K ** 0.5
    cs, ss = M.w4_shapes(O, K, group)
    codes, scales = torch.empty(cs, dtype=torch.uint8, device="cuda"), torch.empty(ss, dtype=torch.bfloat16, device="cuda")
    M.minw_pack_w4(w, group, codes, scales)
    down, up = _rand(gen, n, r, K) / 32, _rand(gen, n, r, O) / 4
    ids = torch.tensor([0, 3, -1, 2, 2, 0, 1, 3, 3], dtype=torch.int32, device="cuda")
    xs, ks = [_rand(gen, T, K).to(dt) for _ in range(20)], [scales * 2 ** (k % 3) for k in range(20)]
    x, s = torch.empty(T, ld, dtype=dt, device="cuda")[:, :K], torch.empty_like(scales)
    ws = _scratch(M.minw_adapters_workspace_bytes(T, K, O, n, r), 255)
    want, got = [torch.empty(T, O, device="cuda") for _ in xs], [torch.empty(T, O, device="cuda") for _ in xs]
    for v, k, y in zip(xs, ks, want):
        v = torch.empty(T, ld, dtype=dt, device="cuda")[:, :K].copy_(v)
        torch.cuda.synchronize()
        M.minw_w4_adapters(v, codes, k, group, ids, down, up, y, workspace=_scratch(ws.nbytes, 0))
        torch.cuda.synchronize()
    for v, k, y in zip(xs, ks, got):
        x.copy_(v)
        s.copy_(k)
        M.minw_w4_adapters(x, codes, s, group, ids, down, up, y, workspace=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("count", [1, 5, 16, 17, 40])
def test_lists_of_other_matrices(M, count):
    """Lists of up to 16 and of more matrices, of other sizes and addresses from call to call."""
    gen = torch.Generator(device="cuda").manual_seed(count)
    lists = [[_rand(gen, 70 + (31 * k + 17 * e) % 200, 66 + (13 * k + 29 * e) % 170) for e in range(count)] for k in range(8)]
    most = max(M.minw_orthogonal_workspace_bytes(g) for g in lists)
    want, got = ([[torch.zeros_like(x) for x in g] for g in lists] for _ in range(2))
    for g, o in zip(lists, want):
        M.minw_orthogonalize(g, o, _scratch(most, 0))
        torch.cuda.synchronize()
    ws = _scratch(most, 255)
    torch.cuda.synchronize()
    for _ in range(2):
        for g, o in zip(lists, got):
            M.minw_orthogonalize(M.MatrixList(g), M.MatrixList(o), ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, o in zip(want, got) for a, b in zip(g, o))
    assert M.minw_get_last_device_error() == M.MINW_OK


@pytest.mark.parametrize("shapes", [[(1100, 1300), (40, 90)], [(2300, 2400)], [(300, 400)] * 20])
def test_two_lists_at_once(M, shapes):
    """Two streams, a list and a workspace each, call after call: the same bits as alone."""
    gen = torch.Generator(device="cuda").manual_seed(len(shapes))
    lists = [[_rand(gen, m, n) for m, n in shapes] for _ in range(2)]
    want, got = ([[torch.zeros_like(x) for x in g] for g in lists] for _ in range(2))
    ws = [_scratch(M.minw_orthogonal_workspace_bytes(g), 255) for g in lists]
    for g, o, w in zip(lists, want, ws):
        M.minw_orthogonalize(g, o, w)
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in lists]
    held = [(M.MatrixList(g), M.MatrixList(o)) for g, o in zip(lists, got)]
    for _ in range(4):
        for (g, o), w, s in zip(held, ws, streams):
            M.minw_orthogonalize(g, o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
    assert M.minw_get_last_device_error() == M.MINW_OK


@pytest.mark.parametrize("T", [1, 64, 65, 100])
def test_beside_4_bit_weights_the_least_workspace(M, T):
    """4 O bytes for each row up to the 32nd; nothing behind them is written."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    K, O, n, r, group = 256, 130, 3, 8, 64
    cs, ss = M.w4_shapes(O, K, group)
    codes, scales = torch.empty(cs, dtype=torch.uint8, device="cuda"), torch.empty(ss, dtype=torch.bfloat16, device="cuda")
    M.minw_pack_w4(_rand(gen, O, K) / 16, group, codes, scales)
    down, up, x = _rand(gen, n, r, K) / 16, _rand(gen, n, r, O), _rand(gen, T, K)
    ids = torch.randint(-1, n, (T,), generator=gen, device="cuda").to(torch.int32)
    need = 4 * O * min(T, 32)
    buf = _scratch(need + 4096, 77)
    want, got = torch.empty(T, O, device="cuda"), torch.empty(T, O, device="cuda")
    M.minw_w4_adapters(x, codes, scales, group, ids, down, up, want, workspace=_scratch(1 << 20, 0))
    M.minw_w4_adapters(x, codes, scales, group, ids, down, up, got, workspace=buf[:need])
    assert torch.equal(want, got) and (buf[need:] == 77).all()
