"""A head answers as it was last packed: codes, group norm and bias of one time."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import head
    return head


def test_no_answer_without_packed_weights(H):
    h = H.Head(2, 2, 32, 5, seed=1)
    x, _ = H.synthetic(3, 2, 2, 32, 5, 0)
    with pytest.raises(RuntimeError, match="pack"):
        h.answer(x)


def test_a_step_changes_no_answer_until_the_next_pack(H):
    """Not the old weights between the new group norm and the new bias."""
    h = H.Head(2, 2, 32, 5, seed=1)
    x, labels = H.synthetic(64, 2, 2, 32, 5, 0)
    h.pack()
    before = h.answer(x[:2])
    h.step(x, labels, lr=0.5)
    assert torch.equal(h.answer(x[:2]), before)
    h.pack()
    assert not torch.equal(h.answer(x[:2]), before)
