"""4-bit weights with group scales: packing bit for bit, products against
their definition in 64 bits.

Bound of a product: every product of a code and a (part of an) x is exact; the
tensor cores add them in fp32 in their own order, rounding or truncating, and
a group's sum is scaled and added with one rounding.  Each of the K terms (three
a value for fp32 vectors) and G groups adds at most 2^-23 of the sum of
magnitudes:

  |acc error| <= (3 K + G + 64) 2^-23 sum |x w|

(64 for the sums over warps, blocks and parts), then the epilogue's rounding
and its activation's, as in the group norm's tests."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import oracle as O  # noqa: E402
from paper_2003_04296_gb300.inputs import DEFAULT_THR  # noqa: E402
from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f": torch.float32, "b": torch.bfloat16}


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _unpack(codes, K):
    """Codes [O][K] from the layout's definition, value by value."""
    c = codes.cpu().numpy()
    words = c.reshape(c.shape[0], -1, 16, 4).astype(np.uint32)
    words = words[..., 0] | words[..., 1] << 8 | words[..., 2] << 16 | words[..., 3] << 24
    out = np.empty((c.shape[0], c.shape[1] * 2), dtype=np.int64)
    for k in range(out.shape[1]):
        blk, r = divmod(k, 128)
        j, t, i = r // 32, r % 32 // 8, r % 8
        out[:, k] = (words[:, blk, 4 * t + j] >> (4 * (i // 2 + 4 * (i % 2)))) & 15
    assert (out[:, K:] == 8).all()
    return out[:, :K]


def _empty(M, O_, K, group):
    sc, ss = M.w4_shapes(O_, K, group)
    return (torch.full(sc, 0xEE, dtype=torch.uint8, device="cuda"),
            torch.full(ss, float("nan"), dtype=torch.bfloat16, device="cuda"))


SHAPES = [(1, 1, 32), (3, 7, 64), (5, 32, 32), (4, 33, 32), (9, 128, 128), (7, 129, 64), (2, 130, 128), (6, 1000, 256),
          (3, 300, 1024), (17, 4097, 32), (130, 520, 128)]


@pytest.mark.parametrize("O_,K,group", SHAPES)
@pytest.mark.parametrize("t", ["f", "b"])
def test_pack(M, O_, K, group, t):
    r = np.random.default_rng(case_seed(O_, K, group))
    w = torch.from_numpy((r.standard_normal((O_, K)) * np.exp(r.standard_normal((O_, 1)))).astype(np.float32)).to(DT[t])
    w[0, 0] = 0
    w[-1, : min(K, group)] = 0                                  # a group of zeros
    codes, scales = _empty(M, O_, K, group)
    M.minw_pack_w4(w.cuda(), group, codes, scales)
    wf = w.float().numpy()
    G = (K + group - 1) // group
    pad = np.zeros((O_, G * group), dtype=np.float32)
    pad[:, :K] = wf
    s = torch.from_numpy(np.abs(pad).reshape(O_, G, group).max(2) / np.float32(7)).bfloat16()
    assert torch.equal(scales.cpu(), s)
    d = np.repeat(s.float().numpy(), group, axis=1)[:, :K]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(d > 0, np.clip(np.rint(wf / d), -7, 7), 0).astype(np.int64)
    assert np.array_equal(_unpack(codes, K), q + 8)


@pytest.mark.parametrize("bits", [1, 2, 3])
@pytest.mark.parametrize("scaled", [True, False])
def test_pack_of_the_quantizers_levels(M, bits, scaled):
    r = np.random.default_rng(bits)
    w = r.normal(0, 0.6, (37, 200)).astype(np.float32)
    cs = r.uniform(0.5, 2, 37).astype(np.float32) if scaled else None
    codes, scales = _empty(M, 37, 200, 64)
    M.minw_pack_w4(torch.from_numpy(w).cuda(), 64, codes, scales, q=M.quant(bits, DEFAULT_THR[bits]),
                   channel_scale=None if cs is None else torch.from_numpy(cs).cuda())
    lv = O.quantize(w[:, :, None, None], bits, DEFAULT_THR[bits], cs) * 2.0 ** O.units_shift(bits)
    assert np.array_equal(_unpack(codes, 200) - 8, lv[:, :, 0, 0])
    assert (scales == 1).all()


def test_pack_of_a_group_that_is_no_number(M):
    w = torch.ones(2, 96, device="cuda")
    w[0, 40], w[1, 70] = float("nan"), float("inf")
    codes, scales = _empty(M, 2, 96, 32)
    M.minw_pack_w4(w, 32, codes, scales)
    c, s = _unpack(codes, 96), scales.float().cpu().numpy()
    assert np.isnan(s[0, 1]) and np.isinf(s[1, 2])
    assert (c[0, 32:64] == 8).all() and (c[1, 64:] == 8).all()
    assert (c[0, :32] == 15).all() and (c[1, :64] == 15).all()


def _weights(M, rng, O_, K, group):
    """Codes over all sixteen values and scales, packed by the layout's definition."""
    u = rng.integers(0, 16, (O_, K))
    full = np.full((O_, (K + 127) // 128 * 128), 8)
    full[:, :K] = u
    words = np.zeros((O_, full.shape[1] // 128, 16), dtype=np.uint32)
    for r in range(128):
        j, t, i = r // 32, r % 32 // 8, r % 8
        words[:, :, 4 * t + j] |= full[:, r::128].astype(np.uint32) << np.uint32(4 * (i // 2 + 4 * (i % 2)))
    codes = torch.from_numpy(words.view(np.uint8).reshape(O_, -1).copy()).cuda()
    s = torch.from_numpy(rng.uniform(0.2, 1.8, (O_, (K + group - 1) // group))).bfloat16()
    w = (u - 8) * np.repeat(s.double().numpy(), group, axis=1)[:, :K]
    return codes, s.cuda(), w


# vectors, outputs, length, group, type of x and y, activation, extra row length of x and y
CASES = [
    (1, 1, 1, 32, "b", "f", 0, 0), (1, 3, 5, 128, "f", "f", 0, 0), (1, 16, 128, 128, "b", "b", 0, 0),
    (1, 17, 129, 32, "b", "f", 1, 0), (2, 40, 100, 64, "f", "b", 3, 0), (3, 33, 257, 64, "b", "b", 2, 5),
    (8, 200, 1000, 32, "b", "f", 0, 8), (9, 129, 640, 128, "b", "f", 3, 0), (5, 401, 4097, 32, "f", "f", 0, 0),
    (4, 70, 333, 32, "f", "f", 1, 1), (10, 64, 512, 256, "f", "f", 0, 0), (11, 64, 512, 1024, "f", "f", 0, 0),
    (17, 50, 700, 64, "b", "b", 0, 0), (32, 31, 384, 128, "b", "f", 0, 0), (33, 31, 384, 128, "b", "f", 0, 0),
    (70, 20, 200, 32, "b", "f", 0, 3), (1, 1024, 8192, 128, "b", "f", 1, 0), (1, 5000, 300, 64, "b", "f", 0, 0),
    (1, 40_000, 256, 128, "f", "f", 0, 0), (3, 10_003, 140, 32, "b", "b", 0, 0), (31, 48, 20_000, 128, "b", "f", 0, 0),
    (2, 64, 100_000, 64, "f", "f", 0, 0), (1, 1000, 384, 384, "b", "f", 0, 0),
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("affine", [True, False])
def test_matvec(M, case, affine):
    T, O_, K, group, tx, ty, act, extra = case
    rng = np.random.default_rng(case_seed(*case))
    codes, scales, w = _weights(M, rng, O_, K, group)
    xbuf = torch.full((T, K + extra), float("nan"), dtype=DT[tx], device="cuda")
    x = xbuf[:, extra:] if extra % 2 else xbuf[:, :K]            # odd extras: the rows start off every boundary
    x.copy_(torch.from_numpy(rng.standard_normal((T, K))))
    ybuf = torch.full((T, O_ + extra), 777.0, dtype=DT[ty], device="cuda")
    y = ybuf[:, :O_]
    sc, sh = (rng.uniform(0.5, 1.5, O_).astype(np.float32), rng.standard_normal(O_).astype(np.float32))
    M.minw_w4_matvec(x, codes, scales, group, y, scale=torch.from_numpy(sc).cuda() if affine else None,
                     shift=torch.from_numpy(sh).cuda() if affine else None, act=act)
    if not affine:
        sc, sh = np.ones(O_), np.zeros(O_)
    xd = x.double().cpu().numpy()
    z = xd @ w.T * sc + sh
    mag = np.abs(xd) @ np.abs(w).T * np.abs(sc)
    ref = [z, np.clip(z, -1, 1), np.maximum(z, 0), z / (1 + np.exp(-np.clip(z, -700, None)))][act]
    tz = (3 * K + scales.shape[1] + 64) * 2.0 ** -23 * mag + 2.0 ** -23 * np.abs(z)
    tol = 1.1 * tz + (2 * np.abs(z) + 8) * 2.0 ** -24 * np.abs(ref) + (2.0 ** -8 * np.abs(ref) if ty == "b" else 0) + 1e-30
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= tol).all(), np.max(err / tol)
    assert (ybuf[:, O_:] == 777).all()


@pytest.mark.parametrize("T,O_,K,group,tx", [(1, 100, 1000, 32, "b"), (7, 300, 900, 64, "f"), (1, 64, 5000, 128, "f")])
def test_whole_numbers_are_exact(M, T, O_, K, group, tx):
    """Whole x and scales that are powers of two: every sum is a whole number below 2^24."""
    rng = np.random.default_rng(T + O_)
    codes, scales, _ = _weights(M, rng, O_, K, group)
    u = _unpack(codes, K) - 8
    s = 2.0 ** rng.integers(0, 3, scales.shape)
    x = rng.integers(-9, 10, (T, K))
    y = torch.empty(T, O_, device="cuda")
    M.minw_w4_matvec(torch.from_numpy(x).to(DT[tx]).cuda(), codes, torch.from_numpy(s).bfloat16().cuda(), group, y)
    ref = x @ (u * np.repeat(s, group, axis=1)[:, :K]).T
    assert np.abs(ref).max() < 2 ** 24
    assert np.array_equal(y.cpu().numpy(), ref)


def test_fp32_vectors_keep_their_digits(M):
    """x = 1 + 2^-23 k against weights that cancel its leading part."""
    K = 256
    codes, scales, _ = _weights(M, np.random.default_rng(1), 16, K, 128)
    u = torch.zeros(16, K)
    u[:, 0::2], u[:, 1::2] = 1.0, -1.0
    codes, scales = _empty(M, 16, K, 128)
    M.minw_pack_w4((u * 7).cuda(), 128, codes, scales)
    r = np.random.default_rng(2).integers(0, 1 << 10, K)
    x = (1 + r * 2.0 ** -23).astype(np.float32)[None]
    y = torch.empty(1, 16, device="cuda")
    M.minw_w4_matvec(torch.from_numpy(x).cuda(), codes, scales, 128, y)
    ref = 7 * ((x.astype(np.float64)[0, 0::2] - x.astype(np.float64)[0, 1::2]).sum())
    # the terms are whole multiples of 2^-23: sums of up to 256 leading ones, then of parts below 2^-13
    assert np.abs(y.cpu().numpy() - ref).max() <= 64 * 2.0 ** -23 * 7 * 2.0 ** -13 * K


@pytest.mark.parametrize("tx", ["b", "f"])
def test_infinity_and_nan_stay_in_their_vector(M, tx):
    rng = np.random.default_rng(3)
    codes, scales, w = _weights(M, rng, 33, 200, 64)
    x = torch.from_numpy(rng.standard_normal((4, 200))).to(DT[tx]).cuda()
    clean, y = torch.empty(4, 33, device="cuda"), torch.empty(4, 33, device="cuda")
    M.minw_w4_matvec(x, codes, scales, 64, clean)
    x[1, 199], x[2, 0] = float("inf"), float("nan")
    M.minw_w4_matvec(x, codes, scales, 64, y)
    assert torch.equal(y[[0, 3]], clean[[0, 3]])
    assert torch.isnan(y[2]).all()
    want = np.where(w[:, 199] == 0, np.nan, np.inf * np.sign(w[:, 199]))
    assert np.array_equal(y[1].cpu().numpy(), want, equal_nan=True)


def test_the_weight_only_layer(M):
    """The levels of a 3-bit weight-only fully connected layer: the same products as the tensor-core call's."""
    rng = np.random.default_rng(4)
    T, O_, K = 4, 96, 512
    w = rng.normal(0, 0.5, (O_, K)).astype(np.float32)
    q = M.quant(3, DEFAULT_THR[3])
    codes, scales = _empty(M, O_, K, 128)
    wt = torch.from_numpy(w).cuda()
    M.minw_pack_w4(wt, 128, codes, scales, q=q)
    wb = torch.empty(O_, 1, 1, K, dtype=torch.int16, device="cuda")
    M.minw_pack_weight_bf16(wt.view(O_, K, 1, 1), q, wb)
    x = torch.from_numpy(rng.standard_normal((T, K))).bfloat16().cuda()
    sc, sh = torch.rand(O_, device="cuda") + 0.5, torch.randn(O_, device="cuda")
    a, b = torch.empty(T, O_, device="cuda"), torch.empty(T, O_, 1, 1, device="cuda")
    M.minw_w4_matvec(x, codes, scales, 128, a, scale=sc, shift=sh)
    M.minw_conv2d_bf16(x, T, K, 1, 1, wb, O_, 1, 1, 3, 1, 0, 0, sc, sh, b)
    lv = _unpack(codes, K) - 8
    mag = np.abs(x.double().cpu().numpy()) @ np.abs(lv).T * sc.double().cpu().numpy()
    tol = 2 * ((3 * K + 70) * 2.0 ** -23 * mag + 2.0 ** -22 * np.abs(b.cpu().numpy()).reshape(T, O_))
    assert (np.abs(a.cpu().numpy().astype(np.float64) - b.cpu().numpy().reshape(T, O_)) <= tol).all()


def test_same_bits_on_another_stream(M):
    rng = np.random.default_rng(6)
    codes, scales, _ = _weights(M, rng, 300, 3000, 64)
    x = torch.from_numpy(rng.standard_normal((3, 3000)).astype(np.float32)).cuda()
    a, b = torch.empty(3, 300, device="cuda"), torch.empty(3, 300, device="cuda")
    M.minw_w4_matvec(x, codes, scales, 64, a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(3):
            M.minw_w4_matvec(x, codes, scales, 64, b)
    s.synchronize()
    assert torch.equal(a, b)


def test_no_vector(M):
    codes, scales, _ = _weights(M, np.random.default_rng(7), 8, 64, 32)
    M.minw_w4_matvec(torch.empty(0, 64, device="cuda"), codes, scales, 32, torch.empty(0, 8, device="cuda"))
