"""Group norm with an activation, forward and backward, against its formula
in 64 bits.

Bounds, with u = 2^-24: a mean or a sum of n values merged from partial ones
is within c u of the sum of magnitudes, where c counts the additions a value
takes part in (a thread's run, the rows of a block, the blocks): at most 128 at
these sizes.  So

  |mean error| <= c u max|x|,  |rstd error| / rstd <= c u + (mean error)^2 r^2 / 2
  |z error| <= c u (|gamma| r (max|x| + |x - mean|) + |beta| + |z|)
  |y error| <= 1.1 |z error| + (2 |z| + 8) u |y|      (|act'| <= 1.1; e^-z rounds its argument)
  bf16 outputs add 2^-8 |y|

and for the backward, whose mean and rstd are inputs,

  |dx error| <= c u r (A + mean(A) + |xh| mean(A |xh|)),  A = (|gamma| + e) |dy|
  |dgamma error| <= c u sum (|dy| (1 + e)(|xh| + e)),  |dbeta error| <= c u sum |dy| (1 + e)

with e = |gamma xh| + |beta| + 1 for the error of act'(z) (its second
derivative is at most 1/2) and of xh itself.  Where the derivative jumps
(|z| = 1, z = 0) within the error of z, the test's dy is 0.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

U, C_ADD, EPS = 2.0 ** -24, 128, 1e-5
DT = {"f": torch.float32, "b": torch.bfloat16}


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _act(z, act):
    return [lambda: z, lambda: np.clip(z, -1, 1), lambda: np.maximum(z, 0),
            lambda: z / (1 + np.exp(-z))][act]()


def _dact(z, act):
    s = 1 / (1 + np.exp(-z))
    return [lambda: np.ones_like(z), lambda: (np.abs(z) <= 1) * 1.0, lambda: (z > 0) * 1.0,
            lambda: s * (1 + z * (1 - s))][act]()


def _groups(v, G):
    """[B][P][C] -> [B][G][n] and back."""
    B, P, C = v.shape
    return v.reshape(B, P, G, C // G).transpose(0, 2, 1, 3).reshape(B, G, -1)


def _spread(s, shape, G):
    """A value per image and group at each of its elements."""
    B, P, C = shape
    return np.repeat(s.reshape(B, 1, G), C // G, axis=2) * np.ones((B, P, 1))


def _forward(x, ga, be, G, act):
    g = _groups(x, G)
    m = g.mean(2)
    r = 1 / np.sqrt(((g - m[:, :, None]) ** 2).mean(2) + EPS)
    xh = (x - _spread(m, x.shape, G)) * _spread(r, x.shape, G)
    z = xh * ga + be
    return _act(z, act), m, r, z, xh


def _rows(v, ld, off, dtype):
    """v [B][P][C] on the device as the channels [off, off + C) of rows of ld values; the others hold 777."""
    B, P, C = v.shape
    buf = torch.full((B, P, ld), 777.0, dtype=dtype, device="cuda")
    view = buf[:, :, off:off + C]
    view.copy_(torch.from_numpy(np.ascontiguousarray(v)))
    return buf, view


def _problem(case, offset=0.0):
    B, P, C, G, ld, off, tx, ty, act = case
    rng = np.random.default_rng(case_seed(*case))
    x = rng.standard_normal((B, P, C)) * rng.uniform(0.5, 2, C) + rng.standard_normal(C) + offset
    x = torch.from_numpy(x).to(DT[tx]).double().numpy()
    ga = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    be = (0.2 * rng.standard_normal(C)).astype(np.float32)
    return rng, x, ga, be


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def _ws(M, B, P, C, G, backward=False):
    return torch.empty(max(16, M.minw_group_norm_workspace_bytes(B, P, C, G, backward)), dtype=torch.uint8,
                       device="cuda")


# images, pixels, channels, groups, row length, first channel, types of x and y, activation
CASES = [
    (1, 1, 8, 2, 8, 0, "f", "f", 0),             # one pixel
    (3, 1, 5, 5, 5, 0, "f", "b", 3),             # groups of one value: xh = 0
    (2, 64, 512, 32, 512, 0, "b", "b", 3),       # a small map with wide rows
    (5, 49, 64, 1, 64, 0, "b", "f", 1),          # one group
    (4, 196, 36, 12, 36, 0, "b", "b", 1),        # rows of 72 bytes: 8-byte loads
    (3, 117, 132, 12, 132, 0, "f", "f", 2),      # groups of 11 channels, no vector divides them
    (3, 117, 264, 24, 264, 0, "b", "b", 3),      # the same in eights
    (2, 77, 33, 11, 33, 0, "b", "f", 1),         # odd channels: single loads
    (2, 77, 48, 3, 64, 8, "b", "b", 1),          # channels of a wider row
    (2, 77, 48, 3, 61, 3, "b", "f", 3),          # ... that start and step off every boundary
    (2, 50, 40, 10, 60, 4, "f", "b", 0),
    (37, 64, 128, 32, 128, 0, "f", "b", 1),
    (2, 1024, 128, 32, 128, 0, "f", "b", 3),     # clusters
    (1, 3136, 64, 16, 64, 0, "b", "b", 1),
    (2, 5000, 32, 8, 32, 0, "b", "b", 3),
    (1, 12544, 64, 2, 64, 0, "b", "b", 3),
    (2, 70001, 16, 4, 16, 0, "b", "b", 3),       # an image in several passes
    (1, 70001, 6, 2, 6, 0, "f", "f", 1),
    (1, 30, 2600, 13, 2600, 0, "f", "f", 3),     # more channels than a block has lanes for
    (1, 9, 4104, 1, 4104, 0, "b", "b", 0),
    (1, 9, 1030, 515, 1030, 0, "f", "f", 0),     # hundreds of groups of two
    (300, 4, 24, 4, 24, 0, "f", "f", 2),         # many images
]


def _tol_forward(x, ga, be, G, z, xh, r, y, ty):
    big = _spread(np.abs(_groups(x, G)).max(2), x.shape, G)
    rr = _spread(r, x.shape, G)
    tz = C_ADD * U * (np.abs(ga) * (rr * big + np.abs(xh)) + np.abs(be) + np.abs(z))
    return 1.1 * tz + (2 * np.abs(z) + 8) * U * np.abs(y) + (2.0 ** -8 * np.abs(y) if ty == "b" else 0) + 1e-37


@pytest.mark.parametrize("case", CASES)
def test_forward(M, case):
    B, P, C, G, ld, off, tx, ty, act = case
    _, x, ga, be = _problem(case)
    y_ref, m_ref, r_ref, z, xh = _forward(x, ga.astype(np.float64), be.astype(np.float64), G, act)
    _, xv = _rows(x, ld, off, DT[tx])
    ybuf, yv = _rows(np.zeros_like(x), ld, off, DT[ty])
    mean, rstd = torch.empty(B, G, device="cuda"), torch.empty(B, G, device="cuda")
    M.minw_group_norm(xv, _dev(ga), _dev(be), G, EPS, yv, act=act, mean=mean, rstd=rstd, workspace=_ws(M, B, P, C, G))
    err = np.abs(yv.double().cpu().numpy() - y_ref)
    tol = _tol_forward(x, ga, be, G, z, xh, r_ref, y_ref, ty)
    assert (err <= tol).all(), np.max(err / tol)
    big = np.abs(_groups(x, G)).max(2)
    dm = np.abs(mean.double().cpu().numpy() - m_ref)
    assert (dm <= C_ADD * U * big).all()
    dr = np.abs(rstd.double().cpu().numpy() / r_ref - 1)
    assert (dr <= C_ADD * U * (1 + C_ADD * U * (big * r_ref) ** 2)).all(), dr.max()
    rest = torch.ones(ld, dtype=torch.bool)
    rest[off:off + C] = False
    assert (ybuf[:, :, rest] == 777).all()                     # the rest of the rows is not written


def test_forward_without_affine_or_statistics_and_in_place(M):
    case = (3, 100, 64, 8, 64, 0, "b", "b", 1)
    _, x, _, _ = _problem(case)
    one, zero = np.ones(64), np.zeros(64)
    y_ref, _, r, z, xh = _forward(x, one, zero, 8, 1)
    tol = _tol_forward(x, one, zero, 8, z, xh, r, y_ref, "b")
    _, xv = _rows(x, 64, 0, torch.bfloat16)
    y = torch.empty_like(xv)
    M.minw_group_norm(xv, None, None, 8, EPS, y, act=1, workspace=_ws(M, 3, 100, 64, 8))
    assert (np.abs(y.double().cpu().numpy() - y_ref) <= tol).all()
    M.minw_group_norm(xv, None, None, 8, EPS, xv, act=1, workspace=_ws(M, 3, 100, 64, 8))
    assert torch.equal(xv, y)


@pytest.mark.parametrize("case", [(2, 200, 32, 4, 32, 0, "f", "f", 0), (1, 70001, 8, 2, 8, 0, "f", "f", 0),
                                  (1, 5000, 64, 4, 64, 0, "f", "f", 0)])
def test_a_mean_far_from_zero_costs_no_digits(M, case):
    """Values around 1000 with a spread of about 1: a variance from a sum of squares would lose 20 of fp32's 24 bits."""
    B, P, C, G = case[:4]
    _, x, ga, be = _problem(case, offset=1000.0)
    _, _, r_ref, _, _ = _forward(x, ga, be, G, 0)
    _, xv = _rows(x, C, 0, torch.float32)
    y, mean, rstd = torch.empty_like(xv), torch.empty(B, G, device="cuda"), torch.empty(B, G, device="cuda")
    M.minw_group_norm(xv, _dev(ga), _dev(be), G, EPS, y, mean=mean, rstd=rstd, workspace=_ws(M, B, P, C, G))
    big = np.abs(_groups(x, G)).max(2)
    dr = np.abs(rstd.double().cpu().numpy() / r_ref - 1)
    # an error d of the mean adds d^2 to the variance; the deviations' own rounding is u of each
    assert (dr <= C_ADD * U + (C_ADD * U * big * r_ref) ** 2).all(), dr.max()


@pytest.mark.parametrize("P", [60, 70001])
def test_nan_and_infinity_stay_in_their_group(M, P):
    case = (2, P, 16, 4, 16, 0, "f", "f", 1)
    _, x, ga, be = _problem(case)
    _, clean = _rows(x, 16, 0, torch.float32)
    _, dirty = _rows(x, 16, 0, torch.float32)
    dirty[0, P // 2, 5] = float("nan")          # image 0, group 1
    dirty[1, P - 1, 15] = float("inf")          # image 1, group 3
    ya, yb = torch.empty_like(clean), torch.empty_like(clean)
    for xv, y in ((clean, ya), (dirty, yb)):
        M.minw_group_norm(xv, _dev(ga), _dev(be), 4, EPS, y, act=1, workspace=_ws(M, 2, P, 16, 4))
    hit = torch.zeros_like(ya, dtype=torch.bool)
    hit[0, :, 4:8] = True
    hit[1, :, 12:16] = True
    assert torch.isnan(yb[hit]).all()
    assert torch.equal(ya[~hit], yb[~hit])


# images, pixels, channels, groups, row length, first channel, types of x and dy, activation
BACKWARD = [
    (1, 1, 8, 2, 8, 0, "f", "f", 0),
    (3, 1, 5, 5, 5, 0, "f", "b", 3),
    (2, 64, 512, 32, 512, 0, "b", "b", 3),
    (5, 49, 64, 1, 64, 0, "b", "f", 1),
    (4, 196, 36, 12, 36, 0, "b", "b", 1),
    (3, 117, 132, 12, 132, 0, "f", "f", 2),
    (3, 117, 264, 24, 264, 0, "b", "b", 3),
    (2, 77, 33, 11, 33, 0, "b", "f", 1),
    (2, 77, 48, 3, 61, 3, "b", "b", 3),
    (2, 50, 40, 10, 60, 4, "f", "b", 0),
    (37, 64, 128, 32, 128, 0, "f", "b", 1),
    (2, 1024, 128, 32, 128, 0, "f", "f", 3),
    (2, 3136, 64, 16, 64, 0, "b", "b", 1),
    (1, 12544, 64, 2, 64, 0, "b", "b", 3),
    (2, 70001, 16, 4, 16, 0, "b", "b", 3),
    (1, 70001, 6, 2, 6, 0, "f", "f", 1),
    (1, 30, 2600, 13, 2600, 0, "f", "f", 3),
    (1, 9, 1030, 515, 1030, 0, "f", "f", 0),
    (300, 4, 24, 4, 24, 0, "f", "f", 2),
]


def _backward_problem(M, case):
    B, P, C, G, ld, off, tx, td, act = case
    rng, x, ga, be = _problem(case)
    _, m, r, _, _ = _forward(x, ga, be, G, act)
    m, r = m.astype(np.float32).astype(np.float64), r.astype(np.float32).astype(np.float64)
    xh = (x - _spread(m, x.shape, G)) * _spread(r, x.shape, G)
    z = xh * ga + be
    dy = rng.standard_normal(x.shape)
    big = _spread(r * np.abs(_groups(x, G)).max(2), x.shape, G)
    near = C_ADD * U * (np.abs(ga) * (big + np.abs(xh)) + np.abs(be))
    if act in (1, 2):
        dy[np.abs((np.abs(z) - 1) if act == 1 else z) <= near] = 0
    dy = torch.from_numpy(dy).to(DT[td]).double().numpy()
    return x, ga, be, m, r, xh, z, dy


def _backward_ref(x, ga, r, xh, z, dy, G, act):
    dz = dy * _dact(z, act)
    h = dz * ga
    s1 = _spread(_groups(h, G).mean(2), x.shape, G)
    s2 = _spread(_groups(h * xh, G).mean(2), x.shape, G)
    return _spread(r, x.shape, G) * (h - s1 - xh * s2), (dz * xh).sum((0, 1)), dz.sum((0, 1))


def _run_backward(M, case, x, ga, be, m, r, dy, stream=None):
    B, P, C, G, ld, off, tx, td, act = case
    _, xv = _rows(x, ld, off, DT[tx])
    _, dv = _rows(dy, ld, off, DT[td])
    obuf, ov = _rows(np.zeros_like(x), ld, off, DT[tx])
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    M.minw_group_norm_backward(xv, dv, _dev(ga), _dev(be), _dev(m), _dev(r), G, ov, dgamma=dg, dbeta=db, act=act,
                               workspace=_ws(M, B, P, C, G, True))
    return obuf, ov, dg, db


@pytest.mark.parametrize("case", BACKWARD)
def test_backward(M, case):
    B, P, C, G, ld, off, tx, td, act = case
    x, ga, be, m, r, xh, z, dy = _backward_problem(M, case)
    dx_ref, dg_ref, db_ref = _backward_ref(x, ga, r, xh, z, dy, G, act)
    obuf, ov, dg, db = _run_backward(M, case, x, ga, be, m, r, dy)
    e = np.abs(ga * xh) + np.abs(be) + 1
    A = (np.abs(ga) + e) * np.abs(dy)
    mean = lambda v: _spread(_groups(v, G).mean(2), x.shape, G)                       # noqa: E731
    tol = C_ADD * U * _spread(r, x.shape, G) * (A + mean(A) + np.abs(xh) * mean(A * np.abs(xh))) + 1e-37
    if tx == "b":
        tol = tol + 2.0 ** -8 * np.abs(dx_ref)
    err = np.abs(ov.double().cpu().numpy() - dx_ref)
    assert (err <= tol).all(), np.max(err / tol)
    tg = C_ADD * U * (np.abs(dy) * (1 + e) * (np.abs(xh) + e)).sum((0, 1)) + 1e-37
    tb = C_ADD * U * (np.abs(dy) * (1 + e)).sum((0, 1)) + 1e-37
    eg, eb = np.abs(dg.double().cpu().numpy() - dg_ref), np.abs(db.double().cpu().numpy() - db_ref)
    assert (eg <= tg).all(), np.max(eg / tg)
    assert (eb <= tb).all(), np.max(eb / tb)
    rest = torch.ones(ld, dtype=torch.bool)
    rest[off:off + C] = False
    assert (obuf[:, :, rest] == 777).all()


@pytest.mark.parametrize("P", [64, 96, 100, 128, 160, 200, 256, 400, 512])
@pytest.mark.parametrize("types", ["bb", "bf", "ff"])
def test_backward_of_small_slabs(M, P, types):
    """From a few KB of shared memory per block to more than 48, where a launch has to ask for it."""
    test_backward(M, (2, P, 64, 8, 64, 0, types[0], types[1], 1))


@pytest.mark.parametrize("case", [(150, 1029, 64, 8, 64, 0, "b", "b", 3), (150, 1311, 64, 4, 64, 0, "b", "b", 1),
                                  (80, 1090, 64, 16, 64, 0, "f", "f", 0), (110, 2050, 32, 8, 32, 0, "f", "b", 3),
                                  (130, 1200, 60, 5, 68, 4, "b", "f", 2)])
def test_backward_of_slabs_that_fit_nowhere(M, case):
    """More than the SMs hold at a time: the sums' last pixels are still at hand, the others read again."""
    test_backward(M, case)


@pytest.mark.parametrize("case", [(2, 40, 24, 4, 24, 0, "f", "f", 0), (2, 40, 24, 4, 24, 0, "f", "f", 3),
                                  (1, 1500, 32, 8, 32, 0, "f", "f", 3)])
def test_backward_against_differences(M, case):
    """Along random directions the gradients give the slope of sum(dy act(z)), statistics included: central
    differences of the 64-bit forward, whose own error is below 1e-8 of the terms at this step."""
    B, P, C, G, _, _, _, _, act = case
    rng, x, ga, be = _problem(case)
    dy = rng.standard_normal(x.shape).astype(np.float32).astype(np.float64)
    _, m, r, _, _ = _forward(x, ga, be, G, act)
    _, ov, dg, db = _run_backward(M, case, x, ga, be, m, r, dy)
    f = lambda x_, g_, b_: (dy * _forward(x_, g_, b_, G, act)[0]).sum()               # noqa: E731
    ga, be, h = ga.astype(np.float64), be.astype(np.float64), 1e-5
    for grad, dirs in ((ov, (1, 0, 0)), (dg, (0, 1, 0)), (db, (0, 0, 1))):
        v = rng.standard_normal(x.shape if dirs[0] else (C,))
        slope = (f(x + h * dirs[0] * v, ga + h * dirs[1] * v, be + h * dirs[2] * v)
                 - f(x - h * dirs[0] * v, ga - h * dirs[1] * v, be - h * dirs[2] * v)) / (2 * h)
        terms = grad.double().cpu().numpy() * v
        scale = np.abs(terms).sum() + np.abs(dy).sum()
        assert abs(terms.sum() - slope) <= (C_ADD * U + 1e-8) * scale * 4


def test_backward_in_place_and_without_parameter_gradients(M):
    case = (3, 100, 64, 8, 64, 0, "b", "b", 1)
    x, ga, be, m, r, xh, z, dy = _backward_problem(M, case)
    _, ref, _, _ = _run_backward(M, case, x, ga, be, m, r, dy)
    for at in ("x", "dy"):
        _, xv = _rows(x, 64, 0, torch.bfloat16)
        _, dv = _rows(dy, 64, 0, torch.bfloat16)
        out = xv if at == "x" else dv
        M.minw_group_norm_backward(xv, dv, _dev(ga), _dev(be), _dev(m), _dev(r), 8, out, act=1,
                                   workspace=_ws(M, 3, 100, 64, 8, True))
        assert torch.equal(out, ref)


def test_no_images(M):
    x = torch.empty(0, 5, 8, device="cuda")
    dg, db = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    stat = torch.empty(0, 2, device="cuda")
    M.minw_group_norm(x, None, None, 2, EPS, torch.empty_like(x), mean=None, rstd=None)
    M.minw_group_norm_backward(x, x, None, None, stat, stat, 2, torch.empty_like(x), dgamma=dg, dbeta=db)
    assert (dg == 0).all() and (db == 0).all()


@pytest.mark.parametrize("P", [1024, 70001])
def test_same_bits_on_another_stream(M, P):
    case = (2, P, 32, 4, 32, 0, "b", "b", 3)
    x, ga, be, m, r, xh, z, dy = _backward_problem(M, case)
    _, dx0, dg0, db0 = _run_backward(M, case, x, ga, be, m, r, dy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(3):
            _, dx1, dg1, db1 = _run_backward(M, case, x, ga, be, m, r, dy)
    s.synchronize()
    assert torch.equal(dx0, dx1) and torch.equal(dg0, dg1) and torch.equal(db0, db1)


def test_rows_the_binding_cannot_describe(M):
    x = torch.zeros(2, 6, 8, device="cuda")
    y = torch.empty_like(x)
    for bad in (x.transpose(1, 2), x.expand(2, 6, 8)[:, :, ::2], torch.zeros(4, 6, 8, device="cuda")[::2, :, :]):
        with pytest.raises(ValueError):
            M.minw_group_norm(bad, None, None, 2, EPS, torch.empty(bad.shape, device="cuda"), workspace=_ws(M, 2, 6, 8, 2))
    with pytest.raises(ValueError):
        M.minw_group_norm(x, torch.ones(7, device="cuda"), None, 2, EPS, y, workspace=_ws(M, 2, 6, 8, 2))
    with pytest.raises(M.MinwError):
        M.minw_group_norm(x, None, None, 3, EPS, y, workspace=_ws(M, 2, 6, 8, 2))
