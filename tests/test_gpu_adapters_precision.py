"""What the adapters' products keep of fp32 values; u = 2^-24.

Inputs with one value a row (and adapters with one rank) make
every result a single product a b of fp32 values.  a and b enter as three bf16
parts, what is left after one being 2^-9 of the value and after two 2^-18; the
six products of parts kept are exact and summed smallest first.  Left out: 2 2^-27 +
2^-36 < 0.26 u.  The last addition (2^0 to 2^-8) truncates, below an ulp, 2 u, and a tensor
core may cut the smaller addends at the same place, two of them: 2 u each at most.  Zeros add
nothing after that.  So |error| <= 6.3 u |a b|; a result that enters a second
product (v in the backward) brings its own 6.3 u along, and the rounding of a
multiplication by alpha or of a store u.  Without the products of the third part
the error is up to 3 2^-18 = 192 u: the tests check that their inputs would show that."""
import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f": torch.float32, "b": torch.bfloat16}
U = 2.0 ** -24
ONE = 6.3 * U


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _single(gen, T, C, dtype, at):
    """[T][C] with one value a row, in column at[t]."""
    x = torch.zeros(T, C, device="cuda")
    x[torch.arange(T, device="cuda"), at] = _rand(gen, T)
    return x.to(dtype)


def _parts(v):
    v = v.float()
    p0 = v.bfloat16().float()
    p1 = (v - p0).bfloat16().float()
    return p0.double(), p1.double(), (v - p0 - p1).bfloat16().double()


def _two_parts(a, b):
    """a b without the products of third parts and of two second parts."""
    a0, a1, _ = _parts(a)
    b0, b1, _ = _parts(b)
    return a0 * b0 + a0 * b1 + a1 * b0


def _would_show(a, b, bound, types):
    """Products of low parts matter here: what is left without them is past the bound, where both are fp32."""
    if types == "ff":
        want = a.double() * b.double()
        assert ((_two_parts(a, b) - want).abs() > 2 * bound * want.abs()).any()


def _within(got, want, bound, what):
    bad = (got.double() - want).abs() > bound * want.abs() + 1e-37
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float(((got.double() - want).abs() / (want.abs() + 1e-30)).max() / U)} u"


@pytest.mark.parametrize("T", [1, 7, 40, 100, 300])
@pytest.mark.parametrize("K,O,r", [(1155, 300, 8), (333, 130, 24), (520, 264, 60), (96, 77, 100)])
@pytest.mark.parametrize("types", ["ff", "bf", "fb"])                    # inputs, adapters
@pytest.mark.parametrize("off", [0, 1])
def test_single_products(M, T, K, O, r, types, off):
    tx, tp = (DT[t] for t in types)
    gen = torch.Generator(device="cuda").manual_seed(case_seed(T, K, types))
    n = 3
    ids = (torch.arange(T, device="cuda") % n).to(torch.int32)
    u = ids.long()
    turn = torch.arange(T, device="cuda") // n                            # of a row among its user's: another column each
    # more rows of a user than columns would add up: the later ones get nothing
    kcol, ocol = turn % K, turn % O
    x, dy = _single(gen, T, K, tx, kcol), _single(gen, T, O, tx, ocol)
    x, dy = x * (turn < K)[:, None], dy * (turn < O)[:, None]
    rank = torch.tensor([0, r - 1, r // 2], device="cuda")                # the one rank of a user that is not zero
    only = torch.nn.functional.one_hot(rank, r).bool()[:, :, None]
    if off:                                                               # pools that begin off 16-byte boundaries
        pool = lambda c: torch.empty(n * r * c + 1, dtype=tp, device="cuda")[1:].view(n, r, c)      # noqa: E731
    else:
        pool = lambda c: torch.empty(n, r, c, dtype=tp, device="cuda")                              # noqa: E731
    down, up = pool(K), pool(O)
    down.copy_(_rand(gen, n, r, K) * only)
    up.copy_(_rand(gen, n, r, O) * only)
    ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r, True) + 128 * O, dtype=torch.uint8, device="cuda")
    rows = torch.arange(T, device="cuda")
    y, h = torch.full((T, O), 7.0, device="cuda"), torch.full((T, r), 7.0, device="cuda")
    M.minw_adapters(x, ids, down, up, y, h=h, workspace=ws)
    xv = x[rows, kcol]
    a, b = xv[:, None].expand(T, r), down[u, :, kcol]
    _within(h, a.double() * b.double(), ONE, "h")
    if T >= 40:
        _would_show(a, b, ONE, types)
    hv = h[rows, rank[u]]
    _within(y, hv.double()[:, None] * up[u, rank[u]].double(), ONE + U, "y")
    if T >= 40:
        _would_show(hv[:, None].expand(T, O), up[u, rank[u]], ONE + U, "f" + types[1])
    # backward: v = up dy, dx = down^T v, ddown = v x^T, dup = h dy^T
    hin = _rand(gen, T, r)
    dx, dd, du = torch.full((T, K), 7.0, dtype=tx, device="cuda"), torch.full((n, r, K), 7.0, device="cuda"), torch.full((n, r, O), 7.0, device="cuda")
    M.minw_adapters_backward(x, ids, down, up, hin, dy, ddown=dd, dup=du, dx=dx, workspace=ws)
    dv = dy[rows, ocol]
    v = dv.double() * up[u, rank[u], ocol].double()
    want = v[:, None] * down[u, rank[u]].double()
    _within(dx, want, 2 * ONE + 2 * U if types[0] == "f" else 2.0 ** -8 + 3 * ONE, "dx")
    wd, wu = torch.zeros(n, r, K, dtype=torch.float64, device="cuda"), torch.zeros(n, r, O, dtype=torch.float64, device="cuda")
    wd.index_put_((u, rank[u], kcol), v * xv.double(), accumulate=True)
    wu.index_put_((u[:, None].expand(T, r), torch.arange(r, device="cuda").expand(T, r), ocol[:, None].expand(T, r)),
                  hin.double() * dv.double()[:, None], accumulate=True)
    _within(dd, wd, 2 * ONE + 2 * U, "ddown")
    _within(du, wu, ONE + U, "dup")
