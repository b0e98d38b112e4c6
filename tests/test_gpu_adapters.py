"""Low-rank adapters (forward, beside 4-bit weights, backward) against their
formulas in 64 bits.

Bounds, with u = 2^-24.  A product of fp32 values is up to six products of their
bf16 parts (0 0, 0 1, 1 0, 0 2, 1 1, 2 0), each added to an fp32 sum; a tensor core's
addition truncates, 2 u of what the sum's terms have come to: n products within
12 n u sum|ab|.  What is left out of a product: 2^-9 2^-18 twice and less, below
2^-25; where a bf16 result alone leaves, 3 2^-18 and the left-out ones of the second
matrix product the same, below 2^-15 together.  So with S_h = sum |x down|,
  |dh| <= (12 K + 3) u S_h
  |dz| <= (12 r + 3) u sum|h up| + sum |dh| |up| + the epilogue's three roundings of what it adds,
and every result is rounded by 2^-24 or 2^-8 of itself; SiLU's slope is below 1.1
and its own error 2^-21 of z."""
import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f": torch.float32, "b": torch.bfloat16}
U = 2.0 ** -24
ROUND = {"f": U, "b": 2.0 ** -8}
LEFT_OUT = {True: 3 * U, False: 2.0 ** -15}


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rows_of(x, dtype, pad, off=0):
    """x [T][C] as the first C columns of a wider buffer of 777s."""
    T, C = x.shape
    buf = torch.full((T * (C + pad) + off,), 777.0, dtype=dtype, device="cuda")
    v = buf[off:].view(T, C + pad)[:, :C]
    v.copy_(x)
    return buf, v


def _users(gen, T, n, how):
    if how == "none":
        return torch.full((T,), -1, dtype=torch.int32, device="cuda")
    if how == "one":
        return torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
    ids = torch.randint(-1, n + 1, (T,), generator=gen, device="cuda")          # n: no index either
    if how == "runs":
        ids = ids[torch.cumsum(torch.rand(T, generator=gen, device="cuda") < 0.1, 0).clamp_max(T - 1)]
    ids = torch.where(ids == n, torch.full_like(ids, 2 ** 31 - 1), ids)
    return ids.to(torch.int32)


def _sel(ids, n):
    """Index of each row's adapter (0 for none) and whether it has one."""
    live = (ids >= 0) & (ids < n)
    return torch.where(live, ids, torch.zeros_like(ids)).long(), live[:, None].double()


def _act(z, act):
    return {0: z, 1: z.clamp(-1, 1), 2: z.clamp_min(0), 3: z * torch.sigmoid(z)}[act]


def _forward(x, ids, down, up, alpha, base, scale, shift, act, fine, ty):
    """y, h and the bounds of their errors."""
    n, r, K = down.shape
    u, live = _sel(ids, n)
    x, down, up = x.double(), down.double(), up.double()
    d, p = down[u] * live[:, :, None], up[u] * live[:, :, None]
    al = alpha.double()[u][:, None] if alpha is not None else torch.ones(len(u), 1, device="cuda", dtype=torch.float64)
    h = torch.einsum("tk,trk->tr", x, d)
    eh = (12 * K * U + LEFT_OUT[fine]) * torch.einsum("tk,trk->tr", x.abs(), d.abs())
    t = al * torch.einsum("tr,tro->to", h, p)
    mag = al.abs() * torch.einsum("tr,tro->to", h.abs(), p.abs())
    et = (12 * r * U + LEFT_OUT[fine] + U) * mag + al.abs() * torch.einsum("tr,tro->to", eh, p.abs())
    b = base.double() if base is not None else torch.zeros_like(t)
    s = scale.double() if scale is not None else 1.0
    f = shift.double() if shift is not None else 0.0
    z = (t + b) * s + f
    ez = (et + U * (t + b).abs() + U * et) * (s.abs() if scale is not None else 1.0) + U * z.abs()
    y = _act(z, act)
    ey = 1.1 * ez + (2.0 ** -21 * z.abs() if act == 3 else 0) + ROUND[ty] * y.abs() + ROUND[ty] * 1.1 * ez
    return y, h, ey, eh


def _check(got, want, bound, what):
    bad = (got.double() - want).abs() > bound + 1e-37
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float(((got.double() - want).abs() - bound).max())}"


# T, K, O, n, r, users
SIZES = [
    (1, 8192, 1024, 64, 16, "runs"), (1, 1, 1, 1, 1, "one"), (2, 33, 7, 3, 3, "mixed"), (5, 31, 65, 2, 17, "mixed"),
    (16, 64, 64, 40, 8, "mixed"), (17, 100, 130, 4, 33, "mixed"), (32, 257, 63, 3, 64, "runs"), (33, 96, 200, 5, 64, "mixed"),
    (64, 1155, 1001, 5, 12, "runs"), (65, 1155, 1001, 5, 12, "runs"), (77, 40, 72, 300, 16, "mixed"), (300, 128, 96, 2, 32, "one"),
    (130, 64, 64, 3, 256, "mixed"), (40, 70, 65, 2, 100, "mixed"), (1000, 72, 136, 7, 4, "mixed"), (97, 64, 64, 4, 16, "none"),
    (2500, 32, 16, 1200, 2, "mixed"), (3, 64, 64, 4, 16, "none"), (700, 2048, 512, 9, 24, "runs"),
]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("types", ["bbbb", "ffff", "bfbf", "fbfb", "bb-b", "ff-f"])          # x, adapters, base, y
@pytest.mark.parametrize("pad", [0, 3])
def test_forward(M, size, types, pad):
    T, K, O, n, r, how = size
    tx, tp, tb, ty = types
    seed = case_seed(size, types, pad)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    act, with_h = seed % 4, seed % 3 != 0
    ids = _users(gen, T, n, how)
    xbuf, x = _rows_of(_rand(gen, T, K), DT[tx], pad, pad)
    down, up = (_rand(gen, n, r, K) / K ** 0.5).to(DT[tp]), (_rand(gen, n, r, O) / r ** 0.5).to(DT[tp])
    alpha = torch.rand(n, generator=gen, device="cuda") * 2 if seed % 2 else None
    scale, shift = (torch.rand(O, generator=gen, device="cuda") + 0.5, _rand(gen, O)) if seed % 5 else (None, None)
    base = None if tb == "-" else _rows_of(_rand(gen, T, O), DT[tb], pad)[1]
    ybuf, y = _rows_of(torch.zeros(T, O, device="cuda"), DT[ty], pad, pad)
    h = torch.full((T, r), 777.0, device="cuda") if with_h else None
    ws = torch.full((M.minw_adapters_workspace_bytes(T, K, O, n, r),), 255, dtype=torch.uint8, device="cuda")
    call = lambda: M.minw_adapters(x, ids, down, up, y, alpha=alpha, base=base, scale=scale, shift=shift, act=act,  # noqa
                                   h=h, workspace=ws)
    call()
    fine = ty == "f" or with_h
    want, wh, ey, eh = _forward(x, ids, down, up, alpha, base, scale, shift, act, fine, ty)
    _check(y, want, ey, "y")
    if with_h:
        _check(h, wh, eh + U * wh.abs(), "h")
    view = ybuf[pad:].view(T, O + pad)
    assert (view[:, O:] == 777).all() and (ybuf[:pad] == 777).all()
    first = y.clone()
    ws.zero_()
    call()
    assert torch.equal(first, y)                                               # the same bits on every call
    if tb == ty:
        M.minw_adapters(x, ids, down, up, base, alpha=alpha, base=base, scale=scale, shift=shift, act=act, h=h, workspace=ws)
        assert torch.equal(first, base)                                        # in place


def _backward(x, ids, down, up, alpha, h, dy):
    n, r, K = down.shape
    u, live = _sel(ids, n)
    x, down, up, h, dy = (v.double() for v in (x, down, up, h, dy))
    al = alpha.double()[u][:, None] if alpha is not None else torch.ones(len(u), 1, device="cuda", dtype=torch.float64)
    d, p = down[u] * live[:, :, None], up[u] * live[:, :, None]
    O = dy.shape[1]
    v = al * torch.einsum("to,tro->tr", dy, p)
    ev = (12 * O * U + 4 * U) * al.abs() * torch.einsum("to,tro->tr", dy.abs(), p.abs())
    evc = (12 * O * U + LEFT_OUT[False]) * al.abs() * torch.einsum("to,tro->tr", dy.abs(), p.abs())
    dx = torch.einsum("tr,trk->tk", v, d)
    mag = torch.einsum("tr,trk->tk", v.abs(), d.abs())
    edx = {f: (12 * r * U + LEFT_OUT[f]) * mag + torch.einsum("tr,trk->tk", ev if f else evc, d.abs()) for f in (True, False)}
    out = {}
    one = torch.nn.functional.one_hot(u, n).double() * live                     # [T][n]
    rows = one.sum(0)[:, None, None]
    for name, a, ea, z in (("ddown", v, ev, x), ("dup", al * h * live, U * (al * h * live).abs(), dy)):
        g = torch.einsum("tn,tr,tc->nrc", one, a, z)
        m = torch.einsum("tn,tr,tc->nrc", one, a.abs(), z.abs())
        out[name] = g, (12 * rows * U + 3 * U) * m + torch.einsum("tn,tr,tc->nrc", one, ea, z.abs()) + U * g.abs()
    return dx, edx, out


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("types", ["bbb", "fff", "bfb", "fbf", "bbf", "ffb"])               # x, adapters, dy
@pytest.mark.parametrize("pad", [0, 3])
def test_backward(M, size, types, pad):
    T, K, O, n, r, how = size
    if n * r * (K + O) * T > 4e9:
        pytest.skip("the reference would take long")
    tx, tp, ty = types
    seed = case_seed(size, types, pad)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ids = _users(gen, T, n, how)
    x = _rows_of(_rand(gen, T, K), DT[tx], pad)[1]
    dy = _rows_of(_rand(gen, T, O), DT[ty], pad, pad)[1]
    down, up = (_rand(gen, n, r, K) / K ** 0.5).to(DT[tp]), (_rand(gen, n, r, O) / r ** 0.5).to(DT[tp])
    alpha = torch.rand(n, generator=gen, device="cuda") * 2 if seed % 2 else None
    h = _rand(gen, T, r)
    accumulate = seed % 3 == 0
    dx0 = _rand(gen, T, K).to(DT[tx])
    dxbuf, dx = _rows_of(dx0, DT[tx], pad)
    ddown, dup = (torch.full((n, r, C), 777.0, device="cuda") for C in (K, O))
    ws = torch.full((M.minw_adapters_workspace_bytes(T, K, O, n, r, True),), 255, dtype=torch.uint8, device="cuda")
    M.minw_adapters_backward(x, ids, down, up, h, dy, ddown=ddown, dup=dup, dx=dx, alpha=alpha, accumulate=accumulate,
                             workspace=ws)
    want, edx, grads = _backward(x, ids, down, up, alpha, h, dy)
    if accumulate:
        want = want + dx0.double()
    # v is computed with all parts where ddown is asked for
    _check(dx, want, edx[True] + (U + ROUND[tx]) * want.abs() + 2 * U * dx0.double().abs(), "dx")
    for name, got in (("ddown", ddown), ("dup", dup)):
        _check(got, *grads[name], name)
    assert (dxbuf.view(T, K + pad)[:, K:] == 777).all()
    # each by itself, on another stream: the same bits (dx of bf16 alone leaves smaller products out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    d2, u2, x2 = torch.zeros_like(ddown), torch.zeros_like(dup), dx0.clone()
    ws.fill_(3)
    side.wait_stream(torch.cuda.current_stream())
    M.minw_adapters_backward(x, ids, down, up, h, dy, ddown=d2, alpha=alpha, workspace=ws, stream=side)
    M.minw_adapters_backward(x, ids, down, up, h, dy, dup=u2, alpha=alpha, workspace=ws, stream=side)
    M.minw_adapters_backward(x, ids, down, up, None, dy, dx=x2, alpha=alpha, accumulate=accumulate, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(d2, ddown) and torch.equal(u2, dup)
    _check(x2, want, edx[tx == "f"] + (U + ROUND[tx]) * want.abs() + 2 * U * dx0.double().abs(), "dx alone")


def test_gradients_against_differences(M):
    """A step of the loss sum(c y) along each input."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    T, K, O, n, r = 70, 40, 50, 3, 6
    ids = _users(gen, T, n, "mixed")
    x, down, up = _rand(gen, T, K), _rand(gen, n, r, K) / 6, _rand(gen, n, r, O)
    alpha, c = torch.rand(n, generator=gen, device="cuda") + 0.5, _rand(gen, T, O)
    ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r, True) + M.minw_adapters_workspace_bytes(T, K, O, n, r),
                     dtype=torch.uint8, device="cuda")
    h, y = torch.empty(T, r, device="cuda"), torch.empty(T, O, device="cuda")

    def loss(x, down, up):
        M.minw_adapters(x, ids, down, up, y, alpha=alpha, h=h, workspace=ws)
        return float((y.double() * c.double()).sum())

    loss(x, down, up)
    dx, ddown, dup = torch.empty_like(x), torch.empty_like(down), torch.empty_like(up)
    M.minw_adapters_backward(x, ids, down, up, h, c, ddown=ddown, dup=dup, dx=dx, alpha=alpha, workspace=ws)
    for k, g in enumerate((dx, ddown, dup)):
        v = [torch.zeros_like(t) for t in (x, down, up)]
        v[k] = _rand(gen, *g.shape)
        # the loss is linear in each input: a difference of any width is the derivative, off by the sums' rounding
        up_, down_ = (loss(*(t + s * e for t, e in zip((x, down, up), v))) for s in (1.0, -1.0))
        want = float((g.double() * v[k].double()).sum())
        mag = float((y.double().abs() * c.double().abs()).sum()) + abs(up_) + abs(down_)
        assert abs((up_ - down_) / 2 - want) <= (12 * (K + r) + 8) * U * mag * 4


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_non_finite_rows_stay_alone(M, bad):
    gen = torch.Generator(device="cuda").manual_seed(2)
    for T in (9, 90):
        K, O, n, r = 64, 80, 3, 8
        ids = torch.arange(T, device="cuda", dtype=torch.int32) % 4 - 1
        x, down, up = _rand(gen, T, K), _rand(gen, n, r, K), _rand(gen, n, r, O)
        base = _rand(gen, T, O)
        x[4, 7] = bad                                                          # of no user: the row of none
        x[6, 5] = bad                                                          # of user 1
        y, y0 = torch.empty(T, O, device="cuda"), torch.empty(T, O, device="cuda")
        ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r, True), dtype=torch.uint8, device="cuda")
        ws2 = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r), dtype=torch.uint8, device="cuda")
        M.minw_adapters(x, ids, down, up, y, base=base, workspace=ws2)
        clean = torch.where(x.isfinite(), x, torch.zeros_like(x))
        M.minw_adapters(clean, ids, down, up, y0, base=base, workspace=ws2)
        assert torch.equal(y[4], base[4])
        assert not y[6].isfinite().any()
        keep = torch.arange(T, device="cuda") != 6
        assert torch.equal(y[keep], y0[keep])
        h = _rand(gen, T, r)
        dy = _rand(gen, T, O)
        dx, dd, du = torch.empty_like(x), torch.empty_like(down), torch.empty_like(up)
        M.minw_adapters_backward(x, ids, down, up, h, dy, ddown=dd, dup=du, dx=dx, workspace=ws)
        assert dx.isfinite().all() and du.isfinite().all()
        assert dd[0].isfinite().all() and dd[2].isfinite().all() and not dd[1][:, 5].isfinite().any()
        assert dd[1][:, :5].isfinite().all()


def test_other_adapters_of_the_pool_are_not_read_into_results(M):
    """NaN in the adapters of users without rows."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for T in (5, 200):
        K, O, n, r = 70, 90, 6, 5
        ids = torch.full((T,), 2, dtype=torch.int32, device="cuda")
        down, up = torch.full((n, r, K), float("nan"), device="cuda"), torch.full((n, r, O), float("nan"), device="cuda")
        down[2], up[2] = _rand(gen, r, K), _rand(gen, r, O)
        x, y, dy = _rand(gen, T, K), torch.empty(T, O, device="cuda"), _rand(gen, T, O)
        ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r, True) + 4 * T * O, dtype=torch.uint8, device="cuda")
        h = torch.empty(T, r, device="cuda")
        M.minw_adapters(x, ids, down, up, y, h=h, workspace=ws)
        dd, du = torch.full_like(down, 7.0), torch.full_like(up, 7.0)
        M.minw_adapters_backward(x, ids, down, up, h, dy, ddown=dd, dup=du, workspace=ws)
        assert y.isfinite().all()
        for d in (dd, du):
            assert d[2].isfinite().all() and (d[2] != 0).any()
            d[2] = 0
            assert (d == 0).all()


def test_backward_of_no_row(M):
    K, O, n, r = 40, 50, 3, 4
    down, up = torch.ones(n, r, K, device="cuda"), torch.ones(n, r, O, device="cuda")
    dd, du = torch.full_like(down, 7.0), torch.full_like(up, 7.0)
    e = lambda c: torch.empty(0, c, device="cuda")                              # noqa: E731
    ws = torch.empty(M.minw_adapters_workspace_bytes(0, K, O, n, r, True), dtype=torch.uint8, device="cuda")
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    M.minw_adapters_backward(e(K), ids, down, up, e(r), e(O), ddown=dd, dup=du, workspace=ws)
    assert (dd == 0).all() and (du == 0).all()
    M.minw_adapters(e(K), ids, down, up, e(O), workspace=ws)


# ---------------------------------------------------------------------------
# beside 4-bit weights
# ---------------------------------------------------------------------------

def _levels(codes, K):
    b = codes.view(codes.shape[0], -1, 4, 4, 4)
    n = torch.stack((b & 15, b >> 4), dim=-1).flatten(-2)[..., [0, 4, 1, 5, 2, 6, 3, 7]]
    return n.transpose(2, 3).reshape(codes.shape[0], -1)[:, :K].double() - 8


@pytest.mark.parametrize("size", [(1, 8192, 1024, 3, 16, 128), (6, 512, 300, 100, 16, 64), (10, 129, 17, 2, 5, 32),
                                  (11, 1000, 65, 4, 40, 128), (32, 256, 64, 40, 8, 32), (33, 640, 130, 5, 64, 256),
                                  (100, 200, 70, 3, 12, 64)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("types", ["bbb", "fff", "bfb", "fbf"])                              # x, adapters, y
@pytest.mark.parametrize("pad", [0, 3])
def test_w4(M, size, types, pad):
    T, K, O, n, r, group = size
    tx, tp, ty = types
    seed = case_seed(size, types)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    act = seed % 4
    ids = _users(gen, T, n, "mixed")
    x = _rows_of(_rand(gen, T, K), DT[tx], pad)[1]
    w = _rand(gen, O, K) / K ** 0.5
    shapes = M.w4_shapes(O, K, group)
    codes, scales = torch.empty(shapes[0], dtype=torch.uint8, device="cuda"), torch.empty(shapes[1], dtype=torch.bfloat16, device="cuda")
    M.minw_pack_w4(w, group, codes, scales)
    down, up = (_rand(gen, n, r, K) / K ** 0.5).to(DT[tp]), (_rand(gen, n, r, O) / r ** 0.5).to(DT[tp])
    alpha = torch.rand(n, generator=gen, device="cuda") * 2
    scale, shift = torch.rand(O, generator=gen, device="cuda") + 0.5, _rand(gen, O)
    ybuf, y = _rows_of(torch.zeros(T, O, device="cuda"), DT[ty], pad)
    ws = torch.full((M.minw_adapters_workspace_bytes(T, K, O, n, r),), 255, dtype=torch.uint8, device="cuda")
    call = lambda: M.minw_w4_adapters(x, codes, scales, group, ids, down, up, y, alpha=alpha, scale=scale, shift=shift,  # noqa
                                      act=act, workspace=ws)
    call()
    wd = _levels(codes, K) * scales.double().repeat_interleave(group, 1)[:, :K]
    base = x.double() @ wd.T
    want, _, ey, _ = _forward(x, ids, down, up, alpha, base, scale, shift, act, True, ty)
    eb = (2 * K + 8) * U * (x.double().abs() @ wd.abs().T)
    _check(y, want, ey + 1.2 * eb * scale.double(), "y")
    assert (ybuf.view(T, O + pad)[:, O:] == 777).all()
    first = y.clone()
    for _ in range(3):
        call()
    assert torch.equal(first, y)
    # without adapters: the product alone
    ids.fill_(-1)
    call()
    y2 = torch.empty_like(y)
    M.minw_w4_matvec(x, codes, scales, group, y2, scale=scale, shift=shift, act=act)
    if T <= (32 if tx == "b" else 10):
        assert torch.equal(y, y2)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def test_a_step_of_the_adapters_captured_and_replayed(M):
    """Forward, backward and the orthogonalised step of the pools in one graph, on another stream, against eager calls."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    T, K, O, n, r = 150, 192, 96, 4, 8
    ids = _users(gen, T, n, "runs")
    x, target = _rand(gen, T, K).bfloat16(), _rand(gen, T, O)
    down, up = _rand(gen, n, r, K) / K ** 0.5, torch.zeros(n, r, O, device="cuda")
    mom = [torch.zeros_like(down), torch.zeros_like(up)]
    base = _rand(gen, T, O)
    y, dy, h = torch.empty(T, O, device="cuda"), torch.empty(T, O, device="cuda"), torch.empty(T, r, device="cuda")
    dd, du = torch.empty_like(down), torch.empty_like(up)
    ws = torch.empty(max(M.minw_adapters_workspace_bytes(T, K, O, n, r, b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    wl, ml, gl = (M.MatrixList([t for pair in zip(a.unbind(), b.unbind()) for t in pair])
                  for a, b in ((down, up), mom, (dd, du)))
    wo = torch.empty(M.minw_orthogonal_workspace_bytes(gl), dtype=torch.uint8, device="cuda")

    def step():
        M.minw_adapters(x, ids, down, up, y, base=base, h=h, workspace=ws)
        torch.sub(y, target, out=dy)
        M.minw_adapters_backward(x, ids, down, up, h, dy, ddown=dd, dup=du, workspace=ws)
        M.minw_sgd_orthogonal(wl, ml, gl, 0.05, wo)

    state = [t.clone() for t in (down, up, *mom)]
    for _ in range(3):
        step()
    want = [t.clone() for t in (down, up, *mom, y)]
    for t, s in zip((down, up, *mom), state):
        t.copy_(s)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, (down, up, *mom, y)):
        assert torch.equal(a, b)
    assert M.minw_get_last_device_error() == M.MINW_OK


def test_without_dependent_launches(M):
    gen = torch.Generator(device="cuda").manual_seed(9)
    T, K, O, n, r = 90, 100, 110, 3, 9
    ids = _users(gen, T, n, "mixed")
    x, down, up = _rand(gen, T, K), _rand(gen, n, r, K), _rand(gen, n, r, O)
    ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r), dtype=torch.uint8, device="cuda")
    a, b = torch.empty(T, O, device="cuda"), torch.empty(T, O, device="cuda")
    M.minw_adapters(x, ids, down, up, a, workspace=ws)
    old = M.get_plan_options()
    try:
        M.set_plan_options(pdl=0)
        M.minw_adapters(x, ids, down, up, b, workspace=ws)
    finally:
        M.set_plan_options(old)
    assert torch.equal(a, b)


@pytest.mark.parametrize("T", [60, 2200])
def test_rows_past_32_bits(M, T):
    """Rows so far apart that they pass 2^31 values and 2^32 bytes."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    K, O, n, r, ld = 72, 90, 3, 5, (1 << 32) // T // 8 * 8
    ids = _users(gen, T, n, "mixed")
    xbuf, ybuf = (torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld) for _ in range(2))
    x, y = xbuf[:, 16:16 + K], ybuf[:, 3:3 + O]
    x.copy_(_rand(gen, T, K))
    down, up = _rand(gen, n, r, K) / K ** 0.5, _rand(gen, n, r, O)
    h = torch.empty(T, r, device="cuda")
    ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r, True), dtype=torch.uint8, device="cuda")
    M.minw_adapters(x, ids, down, up, y, h=h, workspace=ws)
    want, wh, ey, eh = _forward(x.contiguous(), ids, down, up, None, None, None, None, 0, True, "b")
    _check(y.contiguous(), want, ey, "y")
    _check(h, wh, eh + U * wh.abs(), "h")
    # backward: dy where y was, dx in the other buffer
    dx, dd, du = xbuf[:, 1000:1000 + K], torch.empty_like(down), torch.empty_like(up)
    M.minw_adapters_backward(x, ids, down, up, h, y, ddown=dd, dup=du, dx=dx, workspace=ws)
    wx, edx, grads = _backward(x.contiguous(), ids, down, up, None, h, y.contiguous())
    _check(dx.contiguous(), wx, edx[True] + (U + ROUND["b"]) * wx.abs(), "dx")
    for name, got in (("ddown", dd), ("dup", du)):
        _check(got, *grads[name], name)


def test_pools_past_32_bits(M):
    """The last adapter of a pool of more than 2^31 values."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    K, O, r = 1 << 16, 40, 16
    n = (1 << 31) // (r * K) + 3
    down = torch.empty((n, r, K), dtype=torch.bfloat16, device="cuda")
    up = _rand(gen, n, r, O).bfloat16()
    for T in (3, 100):
        ids = torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
        down[n - 1].copy_(_rand(gen, r, K) / K ** 0.5)
        x, y = _rand(gen, T, K).bfloat16(), torch.empty(T, O, device="cuda")
        ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r), dtype=torch.uint8, device="cuda")
        M.minw_adapters(x, ids, down, up, y, workspace=ws)
        want, _, ey, _ = _forward(x, ids - (n - 1), down[n - 1:], up[n - 1:], None, None, None, None, 0, True, "f")
        _check(y, want, ey, "y")


def test_y_with_its_neighbours_written_at_the_same_time(M):
    """Two batches whose rows share sixteens of bytes, on two streams: neither disturbs the other's values."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    T, K, O, n, r = 200, 64, 77, 3, 8
    buf = torch.zeros(T, 2 * O + 1, dtype=torch.bfloat16, device="cuda")
    ys = [buf[:, 1:1 + O], buf[:, 1 + O:1 + 2 * O]]
    down, up = _rand(gen, n, r, K) / 8, _rand(gen, n, r, O)
    args = [(_rand(gen, T, K), _users(gen, T, n, "mixed"), torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r), dtype=torch.uint8,
                                                                       device="cuda"), torch.cuda.Stream()) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for (x, ids, ws, s), y in zip(args, ys):
            M.minw_adapters(x, ids, down, up, y, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for (x, ids, ws, s), y in zip(args, ys):
        alone = torch.empty(T, O, dtype=torch.bfloat16, device="cuda")
        M.minw_adapters(x, ids, down, up, alone, workspace=ws)
        assert torch.equal(alone, y)
    assert (buf[:, 0] == 0).all()
