"""The stream of a call without one: the current stream of the current device."""
import ctypes

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


def _handle(s):
    return ctypes.c_void_p(getattr(s, "value", s)).value


@pytest.mark.parametrize("name", [None, "_cuda_getCurrentRawStream"])
def test_current_stream(M, monkeypatch, name):
    """With and without the function of torch that is no part of its interface."""
    torch.cuda.init()
    if name is not None:
        monkeypatch.delattr(torch._C, name)
    s = torch.cuda.Stream()
    assert _handle(M._stream(None)) == ctypes.c_void_p(torch.cuda.current_stream().cuda_stream).value
    with torch.cuda.stream(s):
        assert _handle(M._stream(None)) == s.cuda_stream
    assert _handle(M._stream(s)) == s.cuda_stream
