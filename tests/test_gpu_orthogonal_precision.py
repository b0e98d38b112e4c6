"""Orthogonalised matrices are about as near to the formula in 64 bits as plain
fp32 products are.

Bound: three times the error of the formula in fp32 torch products, and 1e-6 of the
result's Frobenius norm.  With u = 2^-24: a level's operands are the sums of two fp16
numbers, off by 2^-22 at most, 1.2 u on average (fp32 results of a plain product: 0.3 u
for each of its additions that count).  Tensor cores cut the addends of 16
products and their sum at 2^-25 of the largest: 0.5 2^-25 16 = 4 u of what the few
sums of 32 or 64 of K have come to at the most, after which sums go on to nearest; and
those sums are without the identity's part of Z and Q, which is the larger one.
Five to six u a level against two for plain products, amplified alike."""
import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _ns(x):
    x = x / torch.sqrt((x * x).sum())
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(5):
        a = x @ x.T
        x = 3.4445 * x + (-4.7750 * a + 2.0315 * (a @ a)) @ x
    return x.T if tall else x


def _matrix(gen, m, n, kind):
    x = torch.randn(m, n, generator=gen, device="cuda")
    if kind == "batch":
        s = torch.logspace(0, -2, 64, device="cuda")
        x = (torch.randn(m, 64, generator=gen, device="cuda") * s) @ torch.randn(64, n, generator=gen, device="cuda").relu() / 8 + 0.02 * x
    return x


LISTS = [[(10, 1024)], [(16, 8192)], [(64, 300)], [(33, 3000)], [(100, 130)], [(130, 100)], [(128, 1152)], [(300, 200)], [(256, 2304)],
         [(512, 512)], [(512, 4608)], [(1001, 333)], [(1024, 1024)], [(1024, 8192)], [(2200, 2310)], [(600, 700)] * 12,
         [(2300, 2400), (300, 200), (100, 130), (512, 4608), (700, 1000), (1500, 1600)],
         [(100 + 3 * k, 130 + 5 * k) for k in range(20)], [(600, 700)] * 20]


@pytest.mark.parametrize("shapes", LISTS, ids=lambda s: f"{len(s)}x{s[0][0]}x{s[0][1]}")
@pytest.mark.parametrize("kind", ["batch", "noise"])
@pytest.mark.parametrize("bf16", [False, True])
def test_as_near_as_fp32_products(M, shapes, kind, bf16):
    allowed = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        gen = torch.Generator(device="cuda").manual_seed(case_seed(shapes, kind))
        g = [_matrix(gen, m, n, kind) for m, n in shapes]
        g = [x.bfloat16() for x in g] if bf16 else g
        o = [torch.empty_like(x, dtype=torch.float32) for x in g]
        M.minw_orthogonalize(g, o, torch.empty(M.minw_orthogonal_workspace_bytes(g), dtype=torch.uint8, device="cuda"))
        for x, y in zip(g, o):
            want = _ns(x.double())
            scale = float(want.norm())
            plain = float((_ns(x.float()).double() - want).norm()) / scale
            own = float((y.double() - want).norm()) / scale
            assert own <= 3 * plain + 1e-6, (tuple(x.shape), own, plain)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = allowed


@pytest.mark.parametrize("kind", ["batch", "noise"])
@pytest.mark.parametrize("shapes", [[(10, 1024), (5, 49), (23, 5), (60, 3000), (1100, 1200), (127, 40)],
                                    [(1200, 1300), (16, 300), (2, 7), (64, 64), (33, 500), (100, 90)]])
def test_small_sides_beside_large_matrices(M, shapes, kind):
    """They join the large ones: q X + R X then takes up to 41 times the result from values held in 22 bits and sums rounded to 24,
    2.4 u together, 41 2.4 u = 6e-6 off where plain products have small matrices' few roundings."""
    gen = torch.Generator(device="cuda").manual_seed(case_seed(shapes, kind))
    g = [_matrix(gen, m, n, kind) for m, n in shapes]
    o = [torch.empty_like(x) for x in g]
    M.minw_orthogonalize(g, o, torch.empty(M.minw_orthogonal_workspace_bytes(g), dtype=torch.uint8, device="cuda"))
    for x, y in zip(g, o):
        want = _ns(x.double())
        scale = float(want.norm())
        plain = float((_ns(x).double() - want).norm()) / scale
        assert float((y.double() - want).norm()) / scale <= 3 * plain + 7e-6, tuple(x.shape)
