"""Orthogonalised matrices of more tiles than there are SMs, over all numbers of
stages (three Newton-Schulz steps at most each), against the formula in 64 bits.

Bounds: 1e-4 of the result's Frobenius norm for each stage begun, as derived for
the tests of three and of five steps, and a rounding of 2^-8 where bf16 leaves."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f": torch.float32, "b": torch.bfloat16}
ROUND = {"f": 0.0, "b": 2.0 ** -8}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _ns(g, steps):
    x = g.double()
    x = x / torch.sqrt((x * x).sum())
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        a = x @ x.T
        x = 3.4445 * x - 4.7750 * (a @ x) + 2.0315 * (a @ (a @ x))
    return x.T if tall else x


def _gradient(gen, m, n):
    s = torch.logspace(0, -2, 16, device="cuda")
    x = (torch.randn(m, 16, generator=gen, device="cuda") * s) @ torch.randn(16, n, generator=gen, device="cuda").relu()
    return x + 0.02 * torch.randn(m, n, generator=gen, device="cuda")


def _bound(steps):
    return 1e-4 * -(-steps // 3)


@pytest.mark.parametrize("steps", [3, 4, 6, 7, 8, 10])
@pytest.mark.parametrize("shape", [(2200, 2310), (1100, 5000), (5000, 1100)])
@pytest.mark.parametrize("t", ["f", "b"])
def test_stages(M, steps, shape, t):
    gen = torch.Generator(device="cuda").manual_seed(case_seed(steps, shape, t))
    g = [_gradient(gen, *shape).to(DT[t]), _gradient(gen, 140, 300).to(DT[t])]
    o = [torch.empty_like(x) for x in g]
    ws = torch.full((M.minw_orthogonal_workspace_bytes(g),), 255, dtype=torch.uint8, device="cuda")
    M.minw_orthogonalize(g, o, ws, steps=steps)
    for x, y in zip(g, o):
        want = _ns(x, steps)
        assert float((y.double() - want).norm()) <= (_bound(steps) + ROUND[t]) * float(want.norm())
    first = [x.clone() for x in o]
    ws.zero_()
    M.minw_orthogonalize(g, o, ws, steps=steps)
    assert all(torch.equal(a, b) for a, b in zip(first, o))                # the same bits on every call
    M.minw_orthogonalize(g, g, ws, steps=steps)                            # in place
    assert all(torch.equal(a, b) for a, b in zip(first, g))


@pytest.mark.parametrize("steps", [7, 10])
def test_update_of_many_steps(M, steps):
    gen = torch.Generator(device="cuda").manual_seed(steps)
    m, n, lr, mu = 4000, 1300, 0.25, 0.5
    g, mom, w = _gradient(gen, m, n), _gradient(gen, m, n), torch.rand(m, n, generator=gen, device="cuda")
    m0, w0 = mom.clone(), w.clone()
    ws = torch.empty(M.minw_orthogonal_workspace_bytes([g]), dtype=torch.uint8, device="cuda")
    M.minw_sgd_orthogonal([w], [mom], [g], lr, ws, momentum=mu, nesterov=True, steps=steps)
    wm = mu * m0.double() + g.double()
    assert ((mom.double() - wm).abs() <= U * wm.abs()).all()
    rate, ns = lr * math.sqrt(m / n), _ns(g.double() + mu * wm, steps)
    want = w0.double() - rate * ns
    assert float((w.double() - want).norm()) <= (_bound(steps) + 4 * U) * rate * float(ns.norm()) + 2 * U * float(want.norm())
    assert M.minw_get_last_device_error() == M.MINW_OK
