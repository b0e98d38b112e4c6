"""Lists of gradients whose tensors lie at other offsets than the tensors beside
them (weights, clipped outputs), and the sums' own bounds.

Bounds, with u = 2^-24.  A thread adds up to 32 squares in fp32, in two halves:
16 fused additions each and one of the halves, 17 u.  Those sums are added with
compensation (the rounding of what the compensation gathers is of order u^2 a
term) and in fp64 across blocks, so the sum of squares is within 18 u, the norm
within 9 u for that, u / 2 for the sum as fp32 under the root and u for the root:
11 u.  k = max_norm / norm is within 12 u, k g within 13 u; w - lr k g rounds once
more, and bf16 results to 2^-8 of themselves."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NORM, SCALED = 11 * U, 13 * U
ROUND = {"f": U, "b": 2.0 ** -8}
DT = {"f": torch.float32, "b": torch.bfloat16}
PER = {"f": 4, "b": 8}                   # values of 16 bytes


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _at_offsets(values, dtype, lengths, offsets, per):
    """values as pieces of one buffer, each `offset` values behind a 16-byte boundary, 777 around them."""
    starts, at = [], per
    for n, o in zip(lengths, offsets):
        starts.append(at + o)
        at += -(-(o + n) // per) * per + per
    buf = torch.full((at,), 777.0, dtype=dtype, device="cuda")
    views, i = [], 0
    for n, s in zip(lengths, starts):
        assert buf[s:].data_ptr() % 16 == (s % per) * buf.element_size()
        views.append(buf[s:s + n])
        views[-1].copy_(values[i:i + n])
        i += n
    return buf, views, starts


def _around(buf, lengths, starts):
    keep = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    for n, s in zip(lengths, starts):
        keep[s:s + n] = False
    return bool((buf[keep] == 777).all())


LENGTHS = {"short": [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 31, 40], "chunks": [2047, 2048, 2049, 2055, 2056, 2057, 4099],
           "long": [9001, 70_003]}


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("tg,tw", [("f", "f"), ("f", "b"), ("b", "f"), ("b", "b")])
@pytest.mark.parametrize("clips", [True, False])
def test_every_pair_of_offsets(M, lengths, tg, tw, clips):
    pairs = [(a, b) for a in range(PER[tg]) for b in range(PER[tw])]
    ns = [LENGTHS[lengths][(3 * i + i // 7) % len(LENGTHS[lengths])] for i in range(len(pairs))]
    gen = torch.Generator(device="cuda").manual_seed(case_seed(lengths, tg, tw))
    g = torch.randn(sum(ns), generator=gen, device="cuda").to(DT[tg])
    w = (torch.rand(sum(ns), generator=gen, device="cuda") * 2 - 1).to(DT[tw])
    gbuf, gv, gs = _at_offsets(g, DT[tg], ns, [p[0] for p in pairs], PER[tg])
    wbuf, wv, ws_ = _at_offsets(w, DT[tw], ns, [p[1] for p in pairs], PER[tw])
    ref = float(g.double().square().sum().sqrt())
    max_norm = np.float32(ref * (0.3 if clips else 3.0))
    k = min(1.0, float(max_norm) / ref)
    want = k * g.double()
    norm, ws = torch.empty(1, device="cuda"), torch.empty(M.minw_grad_workspace_bytes(len(ns)), dtype=torch.uint8, device="cuda")
    M.minw_sgd_clip_norm(M.TensorList(wv, 0.875), gv, max_norm, 0.25, norm, ws)
    assert abs(float(norm) - ref) <= NORM * ref
    upd = (w.double() - 0.25 * want).clamp(-0.875, 0.875)
    tol = SCALED * (0.25 * want).abs() + (ROUND[tw] + U) * upd.abs()
    err = (torch.cat(wv).double() - upd).abs()
    assert (err <= tol).all(), float((err / tol).max())
    assert _around(wbuf, ns, ws_) and _around(gbuf, ns, gs)
    if tg != tw:
        return
    obuf, ov, os_ = _at_offsets(torch.zeros_like(g), DT[tg], ns, [p[1] for p in pairs], PER[tg])
    M.minw_grad_clip(gv, ov, max_norm, norm, ws)
    assert abs(float(norm) - ref) <= NORM * ref
    out = torch.cat(ov)
    if not clips:
        assert torch.equal(out, g)
    assert ((out.double() - want).abs() <= (SCALED + ROUND[tg]) * want.abs()).all()
    assert _around(obuf, ns, os_) and torch.equal(torch.cat(gv), g)


def test_a_flat_bucket_and_weights_of_their_own(M):
    """Gradients as the pieces of one buffer with odd lengths, weights allocated one by one: more tensors than one launch
    takes, and a large one."""
    ns = [1_000_003] + [37 + 13 * (i % 91) for i in range(1100)]
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = torch.randn(sum(ns), generator=gen, device="cuda")
    w = [torch.rand(n, generator=gen, device="cuda") for n in ns]
    w0, ref = torch.cat(w).double(), float(g.double().square().sum().sqrt())
    max_norm = np.float32(ref / 2)
    norm, ws = torch.empty(1, device="cuda"), torch.empty(M.minw_grad_workspace_bytes(len(ns)), dtype=torch.uint8, device="cuda")
    M.minw_sgd_clip_norm(w, torch.split(g, ns), max_norm, 0.125, norm, ws)
    step = 0.125 * float(max_norm) / ref * g.double()
    assert abs(float(norm) - ref) <= NORM * ref
    assert ((torch.cat(w).double() - (w0 - step)).abs() <= SCALED * step.abs() + U * (w0 - step).abs()).all()


def test_long_sums_lose_nothing(M):
    """A thread's first sum so large that each later one is below half a unit of it: uncompensated, all of them would be
    lost.  500 M bf16 values; the large ones are the first chunk of 2048 in each of the first 1216 of 2432 shares."""
    n, e = 500_000_000, 0.984375 * 2.0 ** -13
    chunks = -(-n // 2048)
    each = -(-chunks // 2432)
    g = torch.full((n,), e, dtype=torch.bfloat16, device="cuda")
    at = (torch.arange(1216, device="cuda") * (each * 2048))[:, None] + torch.arange(2048, device="cuda")
    g[at.flatten()] = 1.0
    many = at.numel()
    total = many + (n - many) * e * e                        # (exact: few bits each)
    ref = math.sqrt(total)
    # what one such thread's sum would be without compensation
    s, part = np.float32(8 + 24 * e * e), np.float32(32 * e * e)
    parts = 2 * (each // 4) - 1
    for _ in range(parts):
        s = np.float32(s + part)
    assert (8 + 24 * e * e + parts * 32 * e * e - float(s)) / 8 > 3 * NORM
    norm, ws = torch.empty(1, device="cuda"), torch.empty(M.minw_grad_workspace_bytes(1), dtype=torch.uint8, device="cuda")
    M.minw_grad_norm([g], norm, ws)
    assert abs(float(norm) - ref) <= NORM * ref
