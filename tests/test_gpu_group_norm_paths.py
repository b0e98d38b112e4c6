"""Every kernel of the group norm, reached by a shape that takes it, against the
formula in 64 bits (bounds and their derivation: test_gpu_group_norm; a value
takes part in at most 128 additions at these sizes too: at most 58 pixels of a
thread or a channel's rows, 32 rows of a block, 8 blocks, 32 images side by side)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_group_norm as T  # noqa: E402
from tests._norm_paths import backward_cases, forward_cases  # noqa: E402
from tests.test_gpu_group_norm import M  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def _name(c):
    return "-".join(map(str, (*c[1:], c[0][6] + c[0][7])))


@pytest.mark.parametrize("which", forward_cases(), ids=_name)
def test_forward(M, which):  # noqa: F811
    T.test_forward(M, which[0])


@pytest.mark.parametrize("which", backward_cases(), ids=_name)
def test_backward(M, which):  # noqa: F811
    T.test_backward(M, which[0])


# one case of each way, four bf16 values or eight a vector, single values
SOME = [c for c in forward_cases() if c[0][6:8] == ("b", "b") and c[1] != "shared" and c[2:] in ((8, 2), (4, 1), (1, 1))]


@pytest.mark.parametrize("which", SOME, ids=_name)
def test_in_place(M, which):  # noqa: F811
    """y over x: the values read again are the thread's own, not yet replaced."""
    case = which[0]
    B, P, C, G, ld, off, _, _, act = case
    _, x, ga, be = T._problem(case)
    _, xv = T._rows(x, ld, off, torch.bfloat16)
    _, y = T._rows(x, ld, off, torch.bfloat16)
    args = (T._dev(ga), T._dev(be), G, T.EPS)
    M.minw_group_norm(xv, *args, y, act=act, workspace=T._ws(M, B, P, C, G))
    if torch.equal(xv, y):
        raise AssertionError("nothing written")
    M.minw_group_norm(xv, *args, xv, act=act, workspace=T._ws(M, B, P, C, G))
    assert torch.equal(xv, y)


@pytest.mark.parametrize("which", SOME, ids=_name)
def test_nan_and_infinity_stay_in_their_group(M, which):  # noqa: F811
    case = which[0]
    B, P, C, G, ld, off, _, _, act = case
    _, x, ga, be = T._problem(case)
    _, clean = T._rows(x, ld, off, torch.bfloat16)
    _, dirty = T._rows(x, ld, off, torch.bfloat16)
    hit = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    n = C // G
    for b, p, g, v in ((0, P // 2, 1, "nan"), (B - 1, P - 1, G - 1, "inf"), (B // 2, 0, 0, "-inf")):
        dirty[b, p, g * n] = float(v)
        hit[b, :, g * n:(g + 1) * n] = True
    ya, yb = torch.empty_like(clean), torch.empty_like(clean)
    for xv, y in ((clean, ya), (dirty, yb)):
        M.minw_group_norm(xv, T._dev(ga), T._dev(be), G, T.EPS, y, act=act, workspace=T._ws(M, B, P, C, G))
    assert torch.isnan(yb[hit]).all()
    assert torch.equal(ya[~hit], yb[~hit])


@pytest.mark.parametrize("which", [c for c in forward_cases() if c[0][6:8] == ("f", "f") and c[2:] in ((4, 1), (1, 1))], ids=_name)
def test_a_mean_far_from_zero_costs_no_digits(M, which):  # noqa: F811
    """As in test_gpu_group_norm: values around 1000 with a spread of about 1."""
    B, P, C, G, ld, off, _, _, _ = which[0]
    _, x, ga, be = T._problem(which[0], offset=1000.0)
    _, _, r_ref, _, _ = T._forward(x, ga, be, G, 0)
    _, xv = T._rows(x, ld, off, torch.float32)
    y, mean, rstd = torch.empty_like(xv), torch.empty(B, G, device="cuda"), torch.empty(B, G, device="cuda")
    M.minw_group_norm(xv, T._dev(ga), T._dev(be), G, T.EPS, y, mean=mean, rstd=rstd, workspace=T._ws(M, B, P, C, G))
    big = np.abs(T._groups(x, G)).max(2)
    dr = np.abs(rstd.double().cpu().numpy() / r_ref - 1)
    assert (dr <= T.C_ADD * T.U + (T.C_ADD * T.U * big * r_ref) ** 2).all(), dr.max()


BACK = [c for c in backward_cases() if c[0][6:8] == ("b", "b") and c[1] != "shared" and (c[0][3], c[2]) in ((8, 8), (8, 4), (11, 1))]


@pytest.mark.parametrize("which", BACK, ids=_name)
def test_backward_in_place(M, which):  # noqa: F811
    case = which[0]
    B, P, C, G, ld, off, _, _, act = case
    x, ga, be, m, r, xh, z, dy = T._backward_problem(M, case)
    _, ref, dg, db = T._run_backward(M, case, x, ga, be, m, r, dy)
    for at in ("x", "dy"):
        _, xv = T._rows(x, ld, off, torch.bfloat16)
        _, dv = T._rows(dy, ld, off, torch.bfloat16)
        out, pg, pb = xv if at == "x" else dv, torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        M.minw_group_norm_backward(xv, dv, T._dev(ga), T._dev(be), T._dev(m), T._dev(r), G, out, dgamma=pg, dbeta=pb,
                                   act=act, workspace=T._ws(M, B, P, C, G, True))
        assert torch.equal(out, ref) and torch.equal(pg, dg) and torch.equal(pb, db)
