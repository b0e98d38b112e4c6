"""Products with 4-bit weights whose scales begin anywhere: the same bits as on a
16-byte boundary (some blocks' scales then lie on one though the tensor does not)."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import minw
    return minw


@pytest.mark.parametrize("T", [1, 5, 32])
@pytest.mark.parametrize("K,O,group", [(8192, 96, 32), (16384, 40, 128), (16384, 33, 256), (2048, 130, 64), (1000, 20, 32)])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_scales_anywhere(M, T, K, O, group, t):
    gen = torch.Generator(device="cuda").manual_seed(T + K)
    w = torch.randn(O, K, generator=gen, device="cuda") / K ** 0.5
    cs, ss = M.w4_shapes(O, K, group)
    codes, scales = torch.empty(cs, dtype=torch.uint8, device="cuda"), torch.empty(ss, dtype=torch.bfloat16, device="cuda")
    M.minw_pack_w4(w, group, codes, scales)
    x = torch.randn(T, K, generator=gen, device="cuda").to(t)
    want, y = torch.empty(T, O, device="cuda"), torch.empty(T, O, device="cuda")
    M.minw_w4_matvec(x, codes, scales, group, want)
    for off in range(1, 8):
        moved = torch.empty(scales.numel() + off, dtype=torch.bfloat16, device="cuda")[off:].view(ss).copy_(scales)
        M.minw_w4_matvec(x, codes, moved, group, y)
        assert torch.equal(y, want)
