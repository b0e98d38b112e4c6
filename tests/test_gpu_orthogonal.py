"""Orthogonalised matrices and updates against the Newton-Schulz formula in 64
bits.

Bounds, relative to the result's Frobenius norm.  Up to three steps are a
polynomial in A = X X^T (|A| <= 1.447) times X.  With d the error of A: step j
multiplies small singular directions by 3.4445 + b A + c A^2, so an error of A
grows 3.4445^2 = 11.9 times a step, and the factors of j steps together change by
4.775 / 3.4445 (1 + 11.9 + 11.9^2) d = 214 d relative to themselves.  d: operands
of 22 bits make 2^-22 each way; products of 16 are summed by the tensor cores with
truncation for up to 128 of K (eight sums: at most 8 2^-24 of A, whose parts have
one sign on the diagonal, more elsewhere only against larger cancelling parts),
chunks in fp32 to nearest: about 2^-21, so 214 d = 1.0e-4 for each stage of up to
three steps, and errors of later stages add up.  fp32 results: that; bf16
results: their rounding of 2^-8 at most on top."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f": torch.float32, "b": torch.bfloat16}
STAGE = 1e-4
ROUND = {"f": 0.0, "b": 2.0 ** -8}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _ns(g, steps=5):
    """The formula in 64 bits, from the shorter side."""
    x = g.double()
    norm = torch.sqrt((x * x).sum())
    if norm == 0:
        return x
    x = x / norm
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        a = x @ x.T
        x = 3.4445 * x - 4.7750 * (a @ x) + 2.0315 * (a @ (a @ x))
    return x.T if tall else x


def _matrix(gen, m, n, kind="noise"):
    x = torch.randn(m, n, generator=gen, device="cuda")
    if kind == "batch":                                   # a batch's gradient: a few strong directions
        b = 16
        s = torch.logspace(0, -2, b, device="cuda")
        x = (torch.randn(m, b, generator=gen, device="cuda") * s) @ torch.randn(b, n, generator=gen, device="cuda").relu()
        x = x + 0.02 * torch.randn(m, n, generator=gen, device="cuda")
    elif kind == "rank1":
        x = torch.randn(m, 1, generator=gen, device="cuda") @ torch.randn(1, n, generator=gen, device="cuda")
    return x


def _padded(x, dtype, pad, off=0):
    """x with rows `pad` elements wider apart, `off` elements into a buffer of 777s."""
    m, n = x.shape
    buf = torch.full((m * (n + pad) + off,), 777.0, dtype=dtype, device="cuda")
    v = buf[off:].view(m, n + pad)[:, :n]
    v.copy_(x)
    return buf, v


def _gaps_untouched(buf, v, off):
    m, n = v.shape
    ld = v.stride(0) if m > 1 else n
    assert (buf[:off] == 777).all()
    assert (buf[off:].view(m, -1)[:, n:] == 777).all() if m > 1 else (buf[off + ld:] == 777).all()


def _ws(M, grads, fill=255):
    return torch.full((M.minw_orthogonal_workspace_bytes(grads),), fill, dtype=torch.uint8, device="cuda")


def _bound(steps=5):
    return STAGE * -(-steps // 3)


def _close(got, want, t, steps=5):
    got, want = got.double(), want.double()
    scale = float(want.norm())
    if scale == 0:
        assert (got == 0).all()
        return
    assert float((got - want).norm()) <= (_bound(steps) + ROUND[t]) * scale


SHAPES = [
    [(1, 1)], [(1, 200)], [(200, 1)], [(10, 1024)], [(1024, 10)], [(128, 128)], [(129, 127)], [(127, 129), (64, 64)],
    [(256, 1152)], [(1152, 256)], [(333, 1001)], [(700, 700)], [(16, 8192)] * 3 + [(16, 1024)] * 3,
    [(17, 500)], [(500, 33)], [(64, 4096)], [(64, 4097)], [(3, 26000)], [(26000, 16)], [(32, 40), (33, 40), (64, 65), (65, 64), (1, 2)],
    [(128, 27), (128, 1152), (256, 1152), (5, 3), (0, 7), (130, 2304), (2304, 130), (7, 0)], [(1024, 4097)],
]


@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)}x{s[0][0]}x{s[0][1]}")
@pytest.mark.parametrize("types", ["ff", "bb", "bf", "fb"])
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1)])
def test_orthogonalised(M, shapes, types, pad, off):
    gen = torch.Generator(device="cuda").manual_seed(case_seed(shapes, types))
    xs = [_matrix(gen, m, n, "batch" if k % 2 else "noise") if m * n else torch.empty(m, n, device="cuda")
          for k, (m, n) in enumerate(shapes)]
    g = [_padded(x, DT[types[0]], pad, off) for x in xs]
    o = [_padded(torch.zeros_like(x), DT[types[1]], pad, off) for x in xs]
    gv, ov = [v for _, v in g], [v for _, v in o]
    before = [b.clone() for b, _ in g]
    ws = _ws(M, gv)
    M.minw_orthogonalize(gv, ov, ws)
    first = [v.clone() for v in ov]
    for (buf, v), (obuf, out), b in zip(g, o, before):
        assert torch.equal(buf, b)
        if v.numel():
            _close(out, _ns(v), types[1])
            _gaps_untouched(obuf, out, off)
    ws.fill_(0)
    M.minw_orthogonalize(M.MatrixList(gv), M.MatrixList(ov), ws)
    assert all(torch.equal(a, b) for a, b in zip(first, ov))              # the same bits on every call
    if types[0] == types[1]:
        M.minw_orthogonalize(gv, gv, ws)                                  # in place
        assert all(torch.equal(a, b) for a, b in zip(first, gv))


@pytest.mark.parametrize("shape", [(2200, 2310), (2310, 2190), (1100, 5000), (5000, 1100), (1500, 1200)])
@pytest.mark.parametrize("types", ["fb", "bf"])
def test_large(M, shape, types):
    """Enough tiles for blocks in pairs, odd numbers of them."""
    gen = torch.Generator(device="cuda").manual_seed(case_seed(shape, types))
    g = [_matrix(gen, *shape, "batch").to(DT[types[0]]), _matrix(gen, 300, 200).to(DT[types[0]])]
    o = [torch.empty_like(x, dtype=DT[types[1]]) for x in g]
    ws = _ws(M, g)
    M.minw_orthogonalize(g, o, ws)
    first = [x.clone() for x in o]
    for x, y in zip(g, o):
        _close(y, _ns(x), types[1])
    ws.fill_(1)
    M.minw_orthogonalize(g, o, ws)
    assert all(torch.equal(a, b) for a, b in zip(first, o))
    assert M.minw_get_last_device_error() == M.MINW_OK


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7, 10])
@pytest.mark.parametrize("t", ["f", "b"])
def test_steps(M, steps, t):
    gen = torch.Generator(device="cuda").manual_seed(steps)
    g = [_matrix(gen, 150, 420, "batch"), _matrix(gen, 420, 30)]
    o = [torch.empty_like(x, dtype=DT[t]) for x in g]
    M.minw_orthogonalize(g, o, _ws(M, g), steps=steps)
    for x, y in zip(g, o):
        _close(y, _ns(x, steps), t, steps)


@pytest.mark.parametrize("scale", [1e-44, 1e-38, 1e-25, 1e-6, 1e15, 1e30, 1e37])
def test_scale_does_not_matter(M, scale):
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = (_matrix(gen, 90, 300).double().clamp(-3, 3) * scale).float()
    o = torch.empty_like(g)
    M.minw_orthogonalize([g], [o], _ws(M, [g]))
    _close(o, _ns(g), "f")


def test_singular_values_near_one(M):
    gen = torch.Generator(device="cuda").manual_seed(4)
    g = _matrix(gen, 200, 800)
    o = torch.empty_like(g)
    M.minw_orthogonalize([g], [o], _ws(M, [g]))
    s = torch.linalg.svdvals(o.double())
    assert 0.66 < float(s.min()) and float(s.max()) < 1.22


@pytest.mark.parametrize("n", [40, 260])
def test_low_rank_zero_and_non_finite_next_to_ordinary(M, n):
    gen = torch.Generator(device="cuda").manual_seed(6)
    g = [_matrix(gen, 100, n), torch.zeros(100, n, device="cuda"), _matrix(gen, 100, n), _matrix(gen, 100, n),
         _matrix(gen, 100, n, "rank1"), _matrix(gen, 100, n)]
    g[2][99, n - 1] = math.inf
    g[3][5, 0] = math.nan
    o = [torch.empty_like(x) for x in g]
    M.minw_orthogonalize(g, o, _ws(M, g))
    assert (o[1] == 0).all() and o[2].isnan().all() and o[3].isnan().all()
    for k in (0, 4, 5):
        _close(o[k], _ns(g[k]), "f")
    alone = torch.empty_like(g[5])
    M.minw_orthogonalize([g[5]], [alone], _ws(M, [g[5]]))
    _close(alone, _ns(g[5]), "f")


@pytest.mark.parametrize("types", ["ff", "bf", "fb", "bb"])             # gradients, weights
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("momentum", [0.95, 0.0, None])
def test_update(M, types, nesterov, momentum):
    shapes = [(64, 300), (300, 64), (1, 5), (140, 260), (16, 2048)]
    gen = torch.Generator(device="cuda").manual_seed(case_seed(types, nesterov))
    g = [_matrix(gen, m, n, "batch").to(DT[types[0]]) for m, n in shapes]
    m0 = [_matrix(gen, m, n) for m, n in shapes]
    wbuf = [_padded(torch.rand(m, n, generator=gen, device="cuda") * 2 - 1, DT[types[1]], 4, 4) for m, n in shapes]
    w = [v for _, v in wbuf]
    w0 = [v.clone() for v in w]
    mom = [v.clone() for v in m0]
    lr = 0.25
    limits = [0.9, 1.0, math.inf, 0.5, 2.0]
    M.minw_sgd_orthogonal(M.MatrixList(w, limits), None if momentum is None else mom, g, lr, _ws(M, g),
                          momentum=momentum or 0.0, nesterov=nesterov)
    for k, (m, n) in enumerate(shapes):
        u = g[k].double()
        if momentum is not None:
            mu = float(torch.tensor(momentum, dtype=torch.float32))
            want_m = mu * m0[k].double() + u
            # one fused rounding
            assert ((mom[k].double() - want_m).abs() <= U * want_m.abs()).all()
            u = u + mu * want_m if nesterov else want_m
        else:
            assert torch.equal(mom[k], m0[k])
        ns = _ns(u)
        rate = lr * math.sqrt(max(1.0, m / n))
        want = (w0[k].double() - rate * ns).clamp(-limits[k], limits[k])
        err = (w[k].double() - want).norm()
        # the result's bound, the sum's and (bf16) the weight's rounding, the limit's own rounding
        t = types[1]
        tol = (_bound() + 4 * U) * rate * float(ns.norm()) + (2 * U + ROUND[t]) * float(want.norm())
        assert float(err) <= tol
        assert float(w[k].abs().max()) <= torch.tensor(limits[k], dtype=DT[t])
        _gaps_untouched(*wbuf[k], 4)


def test_update_leaves_non_finite_matrices(M):
    g = [torch.randn(30, 50, device="cuda") for _ in range(3)]
    g[1][3, 3] = math.nan
    m = [torch.randn(30, 50, device="cuda") for _ in range(3)]
    m[2][0, 0] = math.inf
    w = [torch.randn(30, 50, device="cuda") for _ in range(3)]
    before = [t.clone() for t in w + m]
    M.minw_sgd_orthogonal(w, m, g, 0.1, _ws(M, g))
    for k in (1, 2):
        assert torch.equal(w[k], before[k]) and torch.equal(m[k], before[3 + k])
    assert not torch.equal(w[0], before[0]) and not torch.equal(m[0], before[3])


def test_many_matrices(M):
    """More than one launch takes."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    g = [_matrix(gen, 1 + k % 40, 1 + (7 * k) % 150) for k in range(500)]
    o = [torch.empty_like(x) for x in g]
    M.minw_orthogonalize(g, o, _ws(M, g))
    for x, y in zip(g, o):
        _close(y, _ns(x), "f")


def test_empty_lists(M):
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    M.minw_orthogonalize([], [], ws)
    M.minw_sgd_orthogonal([], None, [], 0.1, ws)
    M.minw_orthogonalize([torch.empty(0, 4, device="cuda")], [torch.empty(0, 4, device="cuda")], ws)


def test_convolution_weights_as_matrices(M):
    """A tensor of more dimensions counts as [O][the rest]."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    g = torch.randn(48, 32, 3, 3, generator=gen, device="cuda")
    o = torch.empty_like(g)
    M.minw_orthogonalize([g], [o], _ws(M, [g]))
    _close(o.view(48, -1), _ns(g.view(48, -1)), "f")


def test_captured_on_another_stream(M):
    gen = torch.Generator(device="cuda").manual_seed(11)
    g = [_matrix(gen, 60, 700).bfloat16(), _matrix(gen, 300, 200).bfloat16()]
    w = [torch.rand(60, 700, generator=gen, device="cuda"), torch.rand(300, 200, generator=gen, device="cuda")]
    m = [torch.zeros(60, 700, device="cuda"), torch.zeros(300, 200, device="cuda")]
    lists = [M.MatrixList(v) for v in (w, m, g)]
    ws = _ws(M, g)
    w2, m2 = [v.clone() for v in w], [v.clone() for v in m]
    for _ in range(3):
        M.minw_sgd_orthogonal(w2, m2, g, 0.1, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        M.minw_sgd_orthogonal(*lists, 0.1, ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(w + m, w2 + m2))


def test_without_dependent_launches(M):
    """Programmatic launches off: the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    g = [_matrix(gen, 200, 500), _matrix(gen, 20, 500)]
    o, p = [torch.empty_like(x) for x in g], [torch.empty_like(x) for x in g]
    ws = _ws(M, g)
    M.minw_orthogonalize(g, o, ws)
    old = M.get_plan_options()
    try:
        M.set_plan_options(pdl=0)
        M.minw_orthogonalize(g, p, ws)
    finally:
        M.set_plan_options(old)
    assert all(torch.equal(a, b) for a, b in zip(o, p))


def test_no_wait_ran_out(M):
    assert M.minw_get_last_device_error() == M.MINW_OK


@pytest.mark.parametrize("count,extra", [(300, 2), (3, 5), (0, 230)])
def test_small_sides_beside_large_matrices(M, count, extra):
    """Small sides in a launch of their own, with the large ones, and more large ones than a launch takes."""
    gen = torch.Generator(device="cuda").manual_seed(count)
    shapes = [(1 + k % 30, 5 + (11 * k) % 90) for k in range(count)] + [(70 + k % 60, 66 + (3 * k) % 80) for k in range(extra)]
    g = [_matrix(gen, m, n, "batch" if k % 3 else "noise") for k, (m, n) in enumerate(shapes)]
    w, m = [torch.rand_like(x) for x in g], [torch.randn_like(x) for x in g]
    w0, m0 = [x.clone() for x in w], [x.clone() for x in m]
    M.minw_sgd_orthogonal(w, m, g, 0.1, _ws(M, g), momentum=0.5, nesterov=False)
    for k, (a, b) in enumerate(shapes):
        u = 0.5 * m0[k].double() + g[k].double()
        assert ((m[k].double() - u).abs() <= U * u.abs()).all()
        ns = _ns(u)
        want = w0[k].double() - 0.1 * math.sqrt(max(1.0, a / b)) * ns
        # fp32's u of the kernel and the weight's rounding
        tol = (_bound() + 4 * U) * 0.1 * math.sqrt(max(1.0, a / b)) * float(ns.norm()) + 2 * U * float(want.norm())
        assert float((w[k].double() - want).norm()) <= tol, (k, a, b)


def test_rows_past_32_bits(M):
    """Rows 2^20 values apart, past 2^31 values."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    rows = 2200
    gbuf = torch.empty(rows << 20, dtype=torch.bfloat16, device="cuda").view(rows, 1 << 20)
    obuf = torch.empty(rows << 20, dtype=torch.bfloat16, device="cuda").view(rows, 1 << 20)
    for n in (40, 130):
        g, o = gbuf[:, 8:8 + n], obuf[:, 8:8 + n]
        g.copy_(torch.randn(rows, n, generator=gen, device="cuda"))
        M.minw_orthogonalize([g], [o], _ws(M, [g]))
        _close(o.contiguous(), _ns(g.contiguous()), "b")
