"""The head (group norm, clipped updates, 4-bit weights together): its
gradients against autograd of the same formula in 64 bits, its training and its
packed answers.

The two products of the backward and the forward's take bf16 operands: each
differs from the exact product by at most (2^-7 + 2^-16 + K 2^-23) of the sum of
magnitudes, the bound of the library's training products."""
import numpy as np
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


def _forward64(h, x, w):
    """a and logits of the head in 64 bits."""
    B = x.shape[0]
    v = x.double().reshape(B, h.P, h.G, h.C // h.G)
    m = v.mean((1, 3), keepdim=True)
    r = 1 / torch.sqrt(((v - m) ** 2).mean((1, 3), keepdim=True) + 1e-5)
    a = (((v - m) * r).reshape(B, h.P, h.C) * h.gamma.double() + h.beta.double()).clamp(-1, 1).reshape(B, -1)
    return a, a @ w.T + h.bias.double()


def test_step_gradients(H):
    h = H.Head(4, 4, 32, 10, groups=4, seed=3)
    x, labels = H.synthetic(64, 4, 4, 32, 10, 5)
    w0 = h.w.clone()
    a, logits = _forward64(h, x, w0.double())
    loss = h.step(x, labels, lr=0.0)                       # lr 0: the parameters stay
    assert torch.equal(h.w, w0)
    bound = (2.0 ** -7 + 2.0 ** -16 + h.K * 2.0 ** -23)
    dl = bound * (a.abs() @ w0.double().abs().T) + 1e-6     # of the logits
    got = h.buffers[64]["logits"].view(64, 10).double()
    assert ((got - logits).abs() <= dl).all()
    assert abs(float(loss) - float(torch.nn.functional.cross_entropy(logits, labels))) <= 2 * float(dl.max())
    # the weight gradient from the step's own logits: g^T a
    g = torch.softmax(got, 1)
    g[torch.arange(64), labels] -= 1
    g /= 64
    ref = g.T @ a
    tol = (2.0 ** -7 + 2.0 ** -16 + 64 * 2.0 ** -23) * (g.abs().T @ a.abs()) + 1e-7
    assert ((h.grads[0].double() - ref).abs() <= tol).all()
    # the norm is that of all four gradients
    n = torch.sqrt(sum(t.double().square().sum() for t in h.grads))
    assert abs(float(h.norm) - float(n)) <= 1e-5 * float(n)


def test_training_and_packed_answers(H):
    h = H.Head(6, 6, 64, 20, groups=8, w4_group=64, seed=1)
    losses = [float(h.step(*H.synthetic(128, 6, 6, 64, 20, 10 + k))) for k in range(25)]
    assert np.mean(losses[-5:]) < 0.5 * np.mean(losses[:3]), losses
    assert float(h.w.abs().max()) <= 1
    h.pack()
    x, _ = H.synthetic(33, 6, 6, 64, 20, 99)
    one = torch.cat([h.answer(x[i:i + 1]) for i in range(33)])
    assert torch.equal(one[:8], h.answer(x[:8])[:8]) or (one[:8] - h.answer(x[:8])).abs().max() < 1e-4
    # the packed weights' own values, and the rounding of a to bf16
    from tests.test_gpu_w4 import _unpack
    q = torch.from_numpy(_unpack(h.codes, h.K) - 8).cuda().double()
    wq = q * h.scales.double().repeat_interleave(64, dim=1)[:, :h.K]
    a, logits = _forward64(h, x, wq)
    tol = (2.0 ** -8 + 2.0 ** -15 + 4 * h.K * 2.0 ** -23) * (a.abs() @ wq.abs().T) + 1e-5
    assert ((one.double() - logits).abs() <= tol).all()


def test_refusals(H):
    with pytest.raises(ValueError):
        H.Head(3, 3, 10, 5)
    h = H.Head(2, 2, 32, 5)
    x, labels = H.synthetic(32, 2, 2, 32, 5, 0)
    with pytest.raises(ValueError):
        h.step(x, labels)
