"""The global gradient norm, clipping and the clipped update over lists of
tensors, against their formulas in 64 bits.

Bounds, with u = 2^-24: a thread adds at most 128 squares in fp32 and all else
is fp64, so the sum of squares is within 129 u and the norm within 66 u (half of
it, and its own rounding).  k = max_norm / norm is then within 67 u, k g within
68 u, and w - lr k g adds one rounding of the result; bf16 results 2^-8 of
themselves."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests._gpu import case_seed  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f": torch.float32, "b": torch.bfloat16}


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


def _flat(values, dtype, lengths, gap):
    """values as consecutive pieces of one buffer, gap values apart and first: pieces start off every boundary."""
    n = sum(lengths) + gap * (len(lengths) + 1)
    buf = torch.full((n,), 777.0, dtype=dtype, device="cuda")
    views, at, i = [], gap, 0
    for k in lengths:
        views.append(buf[at:at + k])
        views[-1].copy_(values[i:i + k])
        at, i = at + k + gap, i + k
    return buf, views


def _gaps_untouched(buf, lengths, gap):
    at = 0
    for k in lengths + [0]:
        assert (buf[at:at + gap] == 777).all()
        at += gap + k


def _ws(M, n):
    return torch.empty(M.minw_grad_workspace_bytes(n), dtype=torch.uint8, device="cuda")


# lengths, gap, type of gradients, of weights
CASES = [
    ([1], 0, "f", "f"), ([1], 1, "b", "b"), ([0, 3, 0], 1, "f", "f"),
    ([7, 8, 9, 15, 16, 17, 31], 0, "f", "f"), ([7, 8, 9, 15, 16, 17, 31], 1, "b", "b"),
    ([2048, 2049, 2047, 5], 0, "b", "f"), ([2048, 2049, 2047, 5], 3, "f", "b"),
    ([100_003], 1, "f", "f"), ([100_003, 64, 1], 5, "b", "f"),
    ([1_200_000, 17, 40_001], 0, "f", "f"),
    ([30_000_000, 3], 0, "b", "f"),                          # chunks of the largest size, several a block
    ([11] * 100, 1, "f", "f"), ([11 + 7 * (i % 50) for i in range(801)], 0, "f", "f"),   # three capacities, two launches
    ([5] * 1700, 0, "b", "b"),
    ([3000] * 864 + [0] * 200, 0, "f", "f"), ([0] * 900 + [70_000] * 2, 1, "f", "b"), ([9] * 864 + [0, 0, 5, 0], 2, "b", "f"),
]


def _inputs(case):
    lengths, gap, tg, tw = case
    n = sum(lengths)
    gen = torch.Generator(device="cuda").manual_seed(case_seed(n, gap, tg, tw))
    g = torch.randn(n, generator=gen, device="cuda").to(DT[tg])
    w = (torch.rand(n, generator=gen, device="cuda") * 2 - 1).to(DT[tw])
    return g, w


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{sum(c[0])}{c[2]}{c[3]}{c[1]}")
@pytest.mark.parametrize("clips", [True, False])
def test_norm_clip_and_update(M, case, clips):
    lengths, gap, tg, tw = case
    g, w = _inputs(case)
    ref = float(g.double().square().sum().sqrt())
    max_norm = np.float32(ref * (0.3 if clips else 3.0))
    k = min(1.0, float(max_norm) / ref)
    gbuf, gv = _flat(g, DT[tg], lengths, gap)
    wbuf, wv = _flat(w, DT[tw], lengths, gap)
    obuf, ov = _flat(torch.zeros_like(g), DT[tg], lengths, gap)
    norm, ws = torch.full((1,), -1.0, device="cuda"), _ws(M, len(lengths))
    for call in (lambda: M.minw_grad_norm(gv, norm, ws), lambda: M.minw_grad_clip(gv, ov, max_norm, norm, ws),
                 lambda: M.minw_sgd_clip_norm(M.TensorList(wv, 0.9), gv, max_norm, 0.25, norm, ws)):
        norm.fill_(-1)
        call()
        assert abs(float(norm) - ref) <= 66 * U * ref
    rnd = {"f": U, "b": 2.0 ** -8}
    out, new = torch.cat(ov).double(), torch.cat(wv).double()
    want = k * g.double()
    if not clips:
        assert torch.equal(torch.cat(ov), g)
    assert ((out - want).abs() <= (68 * U + rnd[tg]) * want.abs()).all()
    upd = (w.double() - 0.25 * want).clamp(-0.9, 0.9)
    # 0.9 itself is an fp32 number near 0.9
    tol = 70 * U * (0.25 * want).abs() + rnd[tw] * upd.abs() + 2 * U
    assert ((new - upd).abs() <= tol).all()
    for buf in (gbuf, wbuf, obuf):
        _gaps_untouched(buf, lengths, gap)
    # in place
    M.minw_grad_clip(gv, gv, max_norm, norm, ws)
    assert torch.equal(torch.cat(gv), torch.cat(ov))


def test_limits_per_tensor(M):
    w = [torch.full((5,), 0.5, device="cuda"), torch.full((9,), 1.5, device="cuda")]
    g = [torch.full((5,), -10.0, device="cuda"), torch.full((9,), -10.0, device="cuda")]
    norm, ws = torch.empty(1, device="cuda"), _ws(M, 2)
    M.minw_sgd_clip_norm(M.TensorList(w, [1.0, math.inf]), g, 1e6, 0.25, norm, ws)
    assert (w[0] == 1.0).all() and (w[1] == 4.0).all()


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-22, 1e22, 1e30, 3e37])
@pytest.mark.parametrize("t", ["f", "b"])
def test_norm_wherever_it_is_a_number(M, scale, t):
    """Squares far outside fp32's range, next to ordinary gradients and alone."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = (torch.randn(9001, generator=gen, device="cuda", dtype=torch.float64).clamp(-2, 2) * scale * 0.05).to(DT[t])
    norm, ws = torch.empty(1, device="cuda"), _ws(M, 2)
    for views in ([g], [g, torch.ones(3, device="cuda")]):
        ref = math.sqrt(sum(float(v.double().square().sum()) for v in views))
        M.minw_grad_norm(views, norm, ws)
        # a denormal norm has fewer bits
        assert abs(float(norm) - ref) <= 66 * U * ref + 2.0 ** -149


def test_zero_gradients(M):
    z = torch.zeros(100_000, device="cuda")
    w, norm, ws = torch.rand(100_000, device="cuda"), torch.ones(1, device="cuda"), _ws(M, 1)
    w0 = w.clone()
    M.minw_grad_norm([z], norm, ws)
    assert float(norm) == 0
    M.minw_sgd_clip_norm([w], [z], 1.0, 0.1, norm, ws)
    assert torch.equal(w, w0) and float(norm) == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [0, 77_777, 149_999])
def test_a_step_with_a_norm_that_is_no_number_is_skipped(M, bad, at):
    g = torch.ones(150_000, device="cuda")
    g[at] = bad
    parts = [g[:50_001], g[50_001:]]
    w = torch.rand(150_000, device="cuda")
    w0, norm, ws = w.clone(), torch.zeros(1, device="cuda"), _ws(M, 2)
    M.minw_sgd_clip_norm([w[:50_001], w[50_001:]], parts, 1.0, 0.1, norm, ws)
    assert torch.equal(w, w0)
    assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
    out = torch.zeros_like(g)
    M.minw_grad_clip(parts, [out[:50_001], out[50_001:]], 1.0, norm, ws)
    assert torch.equal(out.nan_to_num(3, 4, 5), g.nan_to_num(3, 4, 5))
    M.minw_grad_clip(parts, parts, 1.0, norm, ws)
    assert torch.equal(out.nan_to_num(3, 4, 5), g.nan_to_num(3, 4, 5))


def test_empty_lists(M):
    norm, ws = torch.ones(1, device="cuda"), _ws(M, 0)
    for call in (lambda: M.minw_grad_norm([], norm, ws), lambda: M.minw_grad_clip([], [], 1.0, norm, ws),
                 lambda: M.minw_sgd_clip_norm([], [], 1.0, 0.1, norm, ws),
                 lambda: M.minw_grad_clip([norm[:0]], [norm[:0]], 1.0, norm, ws)):
        norm.fill_(1)
        call()
        assert float(norm) == 0


def test_same_bits_on_another_stream_and_in_a_graph(M):
    g, w = _inputs(([3_000_001, 77], 0, "f", "f"))
    lengths = [3_000_001, 77]
    norm, ws = torch.empty(1, device="cuda"), _ws(M, 2)

    def fresh():
        w1 = w.clone()
        return w1, M.TensorList(torch.split(w1, lengths), 1.0), M.TensorList(torch.split(g, lengths))

    w0, wl, gl = fresh()
    M.minw_sgd_clip_norm(wl, gl, 1.0, 0.1, norm, ws)
    torch.cuda.synchronize()
    n0 = float(norm)
    w1, wl, gl = fresh()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        M.minw_sgd_clip_norm(wl, gl, 1.0, 0.1, norm, ws)
    s.synchronize()
    assert torch.equal(w0, w1) and float(norm) == n0
    w2, wl, gl = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.minw_sgd_clip_norm(wl, gl, 1.0, 0.1, norm, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w0, w2) and float(norm) == n0
