"""Tensors of more than 2^31 values or 2^32 bytes through a head's operators: the
first and last pieces, and those around 2^31, against the formulas in 64 bits.

Bounds as in the operators' own tests with u = 2^-24 and c, the additions a value
takes part in, as these sizes have them.  Forward: a thread merges four pixels at a
time, at most 470 merges of three roundings; c = 2000 covers these and the blocks'.
Backward: a thread adds up to 3720 pixels one by one, an image's chunks and the
images come on top; c = 4500."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U, EPS = 2.0 ** -24, 1e-5
BF = torch.bfloat16


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("80 GB of device memory needed")
    from paper_2003_04296_gb300 import minw
    yield minw
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# three images in chunks (the backward: streaming), many images that are read twice
@pytest.mark.parametrize("B,P", [(3, 11_200_007), (70_001, 480)])
def test_group_norm(M, B, P):
    C, G, act = 64, 8, 3
    assert B * P * C > 2 ** 31
    x = torch.randn((B, P, C), generator=_gen(1), dtype=BF, device="cuda")
    x[:, :, ::3] += 1.5
    ga = 1 + 0.2 * torch.randn(C, generator=_gen(2), device="cuda")
    be = 0.2 * torch.randn(C, generator=_gen(3), device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty((B, G), device="cuda"), torch.empty((B, G), device="cuda")
    ws = torch.empty(max(M.minw_group_norm_workspace_bytes(B, P, C, G, k) for k in (False, True)), dtype=torch.uint8, device="cuda")
    M.minw_group_norm(x, ga, be, G, EPS, y, act=act, mean=mean, rstd=rstd, workspace=ws)
    images = range(B) if B < 10 else [0, 1, 2 ** 31 // (P * C) - 1, 2 ** 31 // (P * C), 2 ** 31 // (P * C) + 1, B - 2, B - 1]
    some = torch.unique(torch.cat([torch.arange(k, min(k + 300, P)) for k in (0, P // 2, max(0, P - 300))])).cuda()
    spread = lambda t: t.repeat_interleave(C // G)                                               # noqa: E731
    for b in images:
        v = x[b].double().view(P, G, C // G)
        m = v.mean((0, 2))
        r = 1 / torch.sqrt((v - m[:, None]).square().mean((0, 2)) + EPS)
        big = v.abs().amax((0, 2))
        assert ((mean[b].double() - m).abs() <= 2000 * U * big).all()
        assert ((rstd[b].double() / r - 1).abs() <= 2000 * U * (1 + 2000 * U * (big * r) ** 2)).all()
        xh = (x[b][some].double() - spread(m)) * spread(r)
        z = xh * ga.double() + be.double()
        ref = z * torch.sigmoid(z)
        tz = 2000 * U * (ga.abs() * (spread(r * big) + xh.abs()) + be.abs() + z.abs())
        assert ((y[b][some].double() - ref).abs() <= 1.1 * tz + (2 * z.abs() + 8) * U * ref.abs() + 2.0 ** -8 * ref.abs()).all()
    # the backward, dy in y's place, dx over it
    dy = y.normal_(generator=_gen(4))
    keep = {b: dy[b].clone() for b in images}
    ref_g, ref_b, mag_g, mag_b = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(4))
    per = max(1, 2 ** 29 // (P * C))
    for b0 in range(0, B, per):
        xh = (x[b0:b0 + per].double() - mean[b0:b0 + per].double().repeat_interleave(C // G, 1)[:, None]) \
            * rstd[b0:b0 + per].double().repeat_interleave(C // G, 1)[:, None]
        z = xh * ga.double() + be.double()
        s = torch.sigmoid(z)
        d = dy[b0:b0 + per].double()
        dz = d * (s * (1 + z * (1 - s)))
        ref_g += (dz * xh).sum((0, 1))
        ref_b += dz.sum((0, 1))
        e = (ga * xh).abs() + be.abs() + 1
        mag_g += (d.abs() * (1 + e) * (xh.abs() + e)).sum((0, 1))
        mag_b += (d.abs() * (1 + e)).sum((0, 1))
        del xh, z, s, d, dz, e
    dga, dbe = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    M.minw_group_norm_backward(x, dy, ga, be, mean, rstd, G, dy, dgamma=dga, dbeta=dbe, act=act, workspace=ws)
    assert ((dga.double() - ref_g).abs() <= 4500 * U * mag_g).all()
    assert ((dbe.double() - ref_b).abs() <= 4500 * U * mag_b).all()
    for b in images:
        r = spread(rstd[b].double())
        xh = (x[b].double() - spread(mean[b].double())) * r
        z = xh * ga.double() + be.double()
        s = torch.sigmoid(z)
        d = keep[b].double()
        h = d * (s * (1 + z * (1 - s))) * ga.double()
        A = (ga.abs() + (ga * xh).abs() + be.abs() + 1) * d.abs()
        group = lambda t: spread(t.view(P, G, C // G).mean((0, 2)))                              # noqa: E731
        s1, s2, a1, a2 = group(h), group(h * xh), group(A), group(A * xh.abs())
        h, xh, A = h[some], xh[some], A[some]
        ref = r * (h - s1 - xh * s2)
        tol = 4500 * U * r * (A + a1 + xh.abs() * a2) + 2.0 ** -8 * ref.abs()
        assert ((dy[b][some].double() - ref).abs() <= tol).all()


def test_gradient_lists(M):
    ns = [2 ** 31 + 12_345, 77]
    g = torch.randn(sum(ns), generator=_gen(5), dtype=BF, device="cuda")
    gv = list(torch.split(g, ns))
    total = sum(float(p.double().square().sum()) for p in torch.split(g, 2 ** 28))
    ref = total ** 0.5
    max_norm = np.float32(ref / 4)
    k = float(max_norm) / ref
    out, norm = torch.zeros_like(g), torch.empty(1, device="cuda")
    ws = torch.empty(M.minw_grad_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    M.minw_grad_clip(gv, torch.split(out, ns), max_norm, norm, ws)
    # (test_gpu_grad_offsets: 11 u; a block's threads add 216 sums each, whose compensation's own rounding is below u)
    assert abs(float(norm) - ref) <= 12 * U * ref
    w = torch.rand(sum(ns), generator=_gen(6), device="cuda")
    pieces = [slice(a, a + 5000) for a in (0, 2 ** 30, 2 ** 31 - 2500, sum(ns) - 5000)]
    w0 = [w[p].double() for p in pieces]
    M.minw_sgd_clip_norm(torch.split(w, ns), gv, max_norm, 0.25, norm, ws)
    for p, old in zip(pieces, w0):
        want = k * g[p].double()
        assert ((out[p].double() - want).abs() <= (14 * U + 2.0 ** -8) * want.abs()).all()
        new = old - 0.25 * want
        assert ((w[p].double() - new).abs() <= 14 * U * (0.25 * want).abs() + U * new.abs()).all()
    # every value was scaled: none left at zero, none unscaled
    for a, b in zip(torch.split(out, 2 ** 28), torch.split(g, 2 ** 28)):
        assert ((a.float() - k * b.float()).abs() <= 2.0 ** -7 * b.float().abs()).all()


def test_w4(M):
    O, K, group = 32_773, 262_272, 128
    cs, ss = M.w4_shapes(O, K, group)
    assert cs[0] * cs[1] > 2 ** 32
    w = torch.randn((O, K), generator=_gen(7), dtype=BF, device="cuda")
    codes = torch.zeros(cs, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(ss, dtype=BF, device="cuda")
    M.minw_pack_w4(w, group, codes, scales)
    edge = 2 ** 32 // cs[1]
    rows = torch.tensor([0, 1, edge // 2, edge - 1, edge, edge + 1, O - 2, O - 1], device="cuda")
    wf = w[rows].float()
    del w
    top = wf.view(len(rows), -1, group).abs().amax(2)
    sc = (top / torch.full_like(top, 7)).to(BF)              # (by a tensor: a true division)
    assert torch.equal(scales[rows], sc)
    d = sc.float().repeat_interleave(group, 1)
    q = torch.where(d > 0, (wf / d).round().clamp(-7, 7), 0).long()
    words = codes[rows].view(torch.int32).view(len(rows), -1, 4, 4).long()                       # [block][t][j]
    nibble = torch.stack([(words >> (4 * (i // 2 + 4 * (i % 2)))) & 15 for i in range(8)], -1)    # [block][t][j][i]
    got = nibble.transpose(2, 3).reshape(len(rows), -1) - 8                                       # 32 j + 8 t + i
    assert torch.equal(got, q)
    x = torch.randn((1, K), generator=_gen(8), dtype=BF, device="cuda")
    y = torch.empty((1, O), device="cuda")
    M.minw_w4_matvec(x, codes, scales, group, y)
    lv = q.double() * sc.double().repeat_interleave(group, 1)
    ref, mag = lv @ x[0].double(), lv.abs() @ x[0].double().abs()
    # (test_gpu_w4's bound a term at every term; here as the sum of a group of 128, of the groups of a warp's share and 64)
    assert ((y[0, rows].double() - ref).abs() <= (128 + ss[1] + 64) * 2.0 ** -23 * mag).all()
    assert (y != 0).all()
