"""What long sums of the adapters keep of their terms, all of one sign; u = 2^-24.

The tensor cores truncate what they add to, for 16 or 32 terms at a time.  a and b enter as
three bf16 parts; left out of a product: 0.26 u.  The sum of so few terms is truncated
after each of its last additions (the smaller parts' come first and are 2^-8 of it at
most): below 6.3 u of it.  These n partial sums are added to nearest,
each addition off by u of the running sum at most, in either direction for random
terms: a standard deviation below u sqrt(n / 3), so 4 u sqrt(n) is 6.9 of them.  A sum
that the tensor cores truncate throughout is off by n u / 2 and more."""
import math

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


def _within(got, want, bound, what):
    bad = (got.double() - want).abs() > bound * want.abs() + 1e-37
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float(((got.double() - want).abs() / (want.abs() + 1e-30)).max() / U)} u"


@pytest.mark.parametrize("T", [3, 100])
@pytest.mark.parametrize("K", [1 << 13, 1 << 17, 1 << 20])
@pytest.mark.parametrize("types", ["ff", "bb", "fb"])
def test_inner_products_of_one_sign(M, T, K, types):
    """Long rows: h over K values."""
    gen = torch.Generator(device="cuda").manual_seed(case_seed(T, K, types))
    n, r, O = 2, 5, 16
    x = torch.rand(T, K, generator=gen, device="cuda").to(DT[types[0]])
    down = torch.rand(n, r, K, generator=gen, device="cuda").to(DT[types[1]])
    up = torch.zeros(n, r, O, dtype=DT[types[1]], device="cuda")
    ids = (torch.arange(T, device="cuda") % n).to(torch.int32)
    y, h = torch.empty(T, O, device="cuda"), torch.empty(T, r, device="cuda")
    ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r), dtype=torch.uint8, device="cuda")
    M.minw_adapters(x, ids, down, up, y, h=h, workspace=ws)
    want = torch.zeros(T, r, dtype=torch.float64, device="cuda")
    for k in range(n):
        want[ids == k] = x[ids == k].double() @ down[k].double().T
    adds = K // 32 // 8 + 16                               # a warp of eight adds up every eighth 32, then warps and blocks
    _within(h, want, ONE + 4 * U * math.sqrt(adds), "h")


@pytest.mark.parametrize("T", [2000, 1 << 15, 1 << 18])
@pytest.mark.parametrize("r", [4, 30, 64])
@pytest.mark.parametrize("types", ["f", "b"])
def test_gradients_of_one_sign(M, T, r, types):
    """One user's many rows: the matrices' gradients over T rows."""
    gen = torch.Generator(device="cuda").manual_seed(case_seed(T, r, types))
    n, K, O = 1, 40, 72
    x, dy = (torch.rand(T, c, generator=gen, device="cuda").to(DT[types]) for c in (K, O))
    h = torch.rand(T, r, generator=gen, device="cuda")
    down, up = (torch.rand(n, r, c, generator=gen, device="cuda").to(DT[types]) for c in (K, O))
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    dd, du = torch.empty(n, r, K, device="cuda"), torch.empty(n, r, O, device="cuda")
    ws = torch.empty(M.minw_adapters_workspace_bytes(T, K, O, n, r, True), dtype=torch.uint8, device="cuda")
    M.minw_adapters_backward(x, ids, down, up, h, dy, ddown=dd, dup=du, workspace=ws)
    v = dy.double() @ up[0].double().T
    adds = T // 16 + 8
    _within(dd[0], v.T @ x.double(), 2 * ONE + 2 * U + 4 * U * math.sqrt(adds) + 4 * U * math.sqrt(20), "ddown")
    _within(du[0], h.double().T @ dy.double(), ONE + U + 4 * U * math.sqrt(adds), "dup")
