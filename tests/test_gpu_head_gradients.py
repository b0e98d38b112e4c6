"""The gradients of a head's step -- gamma, beta, bias, the weights and the input
-- against autograd in 64 bits, from the step's own logits on.

Bounds, with u = 2^-24.  The gradient g of the logits, of magnitude at most 1 / B,
comes from an fp32 softmax: within 64 u / B (arguments below 16 in magnitude,
e^x and a quotient within a few ulp).  The products take bf16 operands and so are
within

  b = 2^-7 + 2^-16 + n 2^-23

of their sum of magnitudes over n terms, the bound of the library's training
products: g_a = g W is off by at most E = (b |g| + 64 u / B) |W|.  HardTanh's mask
may fall either way where z is within its own error of an edge: E there is |g_a|
more.  The norm's backward is linear in what comes in, so E goes through it by
its magnitudes,

  |dx error| <= r (|gamma| E + mean(|gamma| E) + |xh| mean(|gamma| E |xh|))
  |dgamma error| <= sum E |xh|,  |dbeta error| <= sum E

and its own rounding and that of the statistics, c = 128 additions a value as in
test_gpu_group_norm, add c u of the same terms of A = (|gamma| + e) |g_a| with
e = |gamma xh| + |beta| + 1, twice (the sums', the statistics'), with
D = c u (r max|x| + |xh|) for the error of xh."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U, C_ADD, EPS = 2.0 ** -24, 128, 1e-5


@pytest.fixture(scope="module")
def H():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2003_04296_gb300 import head
    return head


# map, channels, classes (no multiple of 64: padded columns; more than 64: two tiles of them), groups, batch
CASES = [(4, 4, 32, 10, 4, 64), (3, 5, 64, 70, 8, 128), (1, 1, 64, 5, 64, 64), (8, 8, 24, 129, 1, 64)]


@pytest.mark.parametrize("Hh,W,C,O,G,B", CASES)
def test_every_gradient(H, Hh, W, C, O, G, B):
    h = H.Head(Hh, W, C, O, groups=G, seed=7)
    gen = torch.Generator(device="cuda").manual_seed(8)
    # parameters that tell gamma's gradient from beta's and the rows of one from another's
    h.gamma.copy_(1 + 0.5 * torch.rand(C, generator=gen, device="cuda"))
    h.beta.copy_(0.3 * torch.randn(C, generator=gen, device="cuda"))
    h.bias.copy_(0.3 * torch.randn(O, generator=gen, device="cuda"))
    x, labels = H.synthetic(B, Hh, W, C, O, 9)
    h.step(x, labels, lr=0.0)                                # lr 0: the parameters stay
    buf = h.buffers[B]
    P, K = h.P, h.K

    logits = buf["logits"].view(B, O).double()
    assert logits.abs().max() < 16
    g = torch.softmax(logits, 1)
    g[torch.arange(B), labels] -= 1
    g /= B
    eg = 64 * U / B

    leaves = [t.double().requires_grad_() for t in (x.view(B, P, C), h.w, h.gamma, h.beta, h.bias)]
    xd, w, ga, be, bias = leaves
    v = xd.unflatten(2, (G, -1))
    m = v.mean((1, 3), keepdim=True)
    r = 1 / torch.sqrt((v - m).square().mean((1, 3), keepdim=True) + EPS)
    xh = ((v - m) * r).flatten(2)
    z = xh * ga + be
    a = z.clamp(-1, 1).reshape(B, K)
    dx, dw, dga, dbe, dbias = torch.autograd.grad((a @ w.T + bias).mul(g).sum(), leaves)

    with torch.no_grad():
        spread = lambda t: t.expand(B, P, G, C // G).flatten(2)                                  # noqa: E731
        mean = lambda t: spread(t.unflatten(2, (G, -1)).mean((1, 3), keepdim=True))              # noqa: E731
        rr, big = spread(r), spread(v.abs().amax((1, 3), keepdim=True))
        bound = lambda n: 2.0 ** -7 + 2.0 ** -16 + n * 2.0 ** -23                                # noqa: E731
        D = C_ADD * U * (rr * big + xh.abs())
        ga_in = (g @ w).view(B, P, C).abs()
        E = ((bound(-(-O // 64) * 64) * g.abs() + eg) @ w.abs()).view(B, P, C)
        edge = (z.abs() - 1).abs() <= ga * D + C_ADD * U * be.abs()
        E = E + edge * ga_in
        e = (ga * xh).abs() + be.abs() + 1
        A = (ga + e) * (ga_in + E)
        own = 2 * C_ADD * U
        tol = rr * (ga * E + mean(ga * E) + xh.abs() * mean(ga * E * xh.abs()))
        tol = tol + own * rr * (A + mean(A) + xh.abs() * mean(A * xh.abs())) + rr * (D * mean(A * xh.abs()) + xh.abs() * mean(A * D))
        err = (buf["dx"].double() - dx).abs()
        assert (err <= tol + 1e-37).all(), float((err / tol).max())
        # (c u a value of a batch's channel sum: at most 128 additions too)
        for got, ref, t in ((h.grads[1], dga, E * xh.abs() + own * A * (xh.abs() + e) + A * D), (h.grads[2], dbe, E + own * A)):
            t = t.sum((0, 1))
            assert ((got.double() - ref).abs() <= t).all(), float(((got.double() - ref).abs() / t).max())
        assert ((h.grads[3].double() - dbias).abs() <= B * eg + B * U * g.abs().sum(0)).all()
        # the weights': a is within D's share of itself
        ta = (bound(B) * g.abs() + eg).T @ a.abs() + g.abs().T @ (ga * D + C_ADD * U * be.abs()).view(B, K)
        assert ((h.grads[0].double() - dw).abs() <= ta).all()
