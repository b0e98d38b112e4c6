"""A classifier head on channels-last feature maps: group norm and HardTanh,
then a fully connected layer.  Trained in small batches (no batch statistics)
with steps clipped by the gradients' global norm, then served one input at a
time from 4-bit weights:

    head = Head(H, W, C, classes)
    loss = head.step(x, labels)              # x [B][H][W][C] on the device, B a multiple of 64
    head.pack()
    logits = head.answer(x1)                 # x1 [T][H][W][C], one input or a few

Every product, norm and update runs in the library; torch holds the tensors
and computes the loss.  ``python -m paper_2003_04296_gb300.head`` trains one on
synthetic classes and compares its packed answers with the trained ones.
"""
import math

import torch

from . import minw

EPS = 1e-5


class Head:
    def __init__(self, H, W, C, classes, groups=8, w4_group=128, seed=0):
        self.P, self.C, self.O, self.G, self.w4_group = H * W, C, classes, groups, w4_group
        self.K = self.P * C
        if self.K % 64 != 0:
            raise ValueError("H W C has to be a multiple of 64")
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.gamma, self.beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        self.bias = torch.zeros(classes, device="cuda")
        self.w = torch.randn((classes, self.K), generator=g, device="cuda").mul_(1 / math.sqrt(self.K))
        self.grads = [torch.empty_like(t) for t in (self.w, self.gamma, self.beta, self.bias)]
        # the latent weights stay in [-1, 1] (Algorithm 1's clip), the others are free
        self.params = minw.TensorList([self.w, self.gamma, self.beta, self.bias],
                                      limits=[1.0, math.inf, math.inf, math.inf])
        self.grad_list = minw.TensorList(self.grads)
        self.norm = torch.empty(1, device="cuda")
        self.grad_ws = self._bytes(minw.minw_grad_workspace_bytes(len(self.grads)))
        self.buffers = {}
        self.codes = self.scales = self.packed = None

    @staticmethod
    def _bytes(n):
        return torch.empty(max(int(n), 16), dtype=torch.uint8, device="cuda")

    def _batch(self, B):
        """Activations, bf16 operands and workspaces of a batch, made once."""
        if B not in self.buffers:
            P, C, O, K = self.P, self.C, self.O, self.K
            f = dict(device="cuda")
            h = dict(dtype=torch.int16, device="cuda")
            Op = (O + 63) // 64 * 64
            self.buffers[B] = dict(
                a=torch.empty((B, P, C), **f), ga=torch.empty((B, K, 1, 1), **f), dx=torch.empty((B, P, C), **f),
                mean=torch.empty((B, self.G), **f), rstd=torch.empty((B, self.G), **f),
                logits=torch.empty((B, O, 1, 1), **f), gw=self.grads[0].view(O, K, 1, 1),
                ab=torch.empty((B, K), **h), atb=torch.empty((K, B), **h), wb=torch.empty((O, K), **h),
                wtb=torch.empty((K, Op), **h), gb=torch.empty((B, Op), **h), gtb=torch.empty((O, B), **h),
                one=torch.ones(max(K, O), **f), zero=torch.zeros(max(K, O), **f),
                ws=self._bytes(minw.minw_group_norm_workspace_bytes(B, P, C, self.G, True)))
        return self.buffers[B]

    def step(self, x, labels, lr=0.1, max_norm=1.0):
        """One training step; returns the loss (on the device).  The input's gradient is left in `dx` of the batch's
        buffers."""
        B, P, C, O, K = x.shape[0], self.P, self.C, self.O, self.K
        if B % 64 != 0:
            raise ValueError("batches of a multiple of 64")
        b = self._batch(B)
        Op = b["gb"].shape[1]
        xr = x.view(B, P, C)
        # forward: a = HardTanh(group norm(x)), logits = a W^T + bias
        minw.minw_group_norm(xr, self.gamma, self.beta, self.G, EPS, b["a"], act=minw.ACT_HARDTANH, mean=b["mean"],
                             rstd=b["rstd"], workspace=b["ws"])
        a = b["a"].view(B, K)
        minw.minw_bf16_matrix(a, b["ab"])
        minw.minw_bf16_matrix(a, b["atb"], transpose=True)
        minw.minw_bf16_matrix(self.w, b["wb"])
        minw.minw_bf16_matrix(self.w, b["wtb"], transpose=True)
        minw.minw_conv2d_bf16(b["ab"], B, K, 1, 1, b["wb"], O, 1, 1, 3, 1, 0, 0, b["one"][:O], self.bias, b["logits"])
        logits = b["logits"].view(B, O)
        loss = torch.nn.functional.cross_entropy(logits, labels)
        g = torch.softmax(logits, dim=1)
        g[torch.arange(B, device="cuda"), labels] -= 1
        g /= B
        # backward: g_W = g^T a, g_a = g W, then through HardTanh and the group norm
        minw.minw_bf16_matrix(g, b["gb"])
        minw.minw_bf16_matrix(g, b["gtb"], transpose=True)
        minw.minw_conv2d_bf16(b["gtb"], O, B, 1, 1, b["atb"], K, 1, 1, 3, 1, 0, 0, b["one"][:K], b["zero"][:K], b["gw"])
        minw.minw_conv2d_bf16(b["gb"], B, Op, 1, 1, b["wtb"], K, 1, 1, 3, 1, 0, 0, b["one"][:K], b["zero"][:K], b["ga"])
        minw.minw_group_norm_backward(xr, b["ga"].view(B, P, C), self.gamma, self.beta, b["mean"], b["rstd"], self.G,
                                      b["dx"], dgamma=self.grads[1], dbeta=self.grads[2], act=minw.ACT_HARDTANH,
                                      workspace=b["ws"])
        torch.sum(g, 0, out=self.grads[3])
        # the clipped update of all parameters
        minw.minw_sgd_clip_norm(self.params, self.grad_list, max_norm, lr, self.norm, self.grad_ws)
        return loss

    def pack(self):
        """The weights as 4-bit codes with a scale per group, and what goes with them as it is now: steps taken later
        change no answer until the next pack()."""
        cs, ss = minw.w4_shapes(self.O, self.K, self.w4_group)
        self.codes = torch.empty(cs, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(ss, dtype=torch.bfloat16, device="cuda")
        minw.minw_pack_w4(self.w, self.w4_group, self.codes, self.scales)
        self.packed = [t.clone() for t in (self.gamma, self.beta, self.bias)]

    def answer(self, x):
        """Logits [T][classes] of one input or a few, from the head as it was packed."""
        if self.packed is None:
            raise RuntimeError("pack() comes before the first answer")
        gamma, beta, bias = self.packed
        T = x.shape[0]
        a = torch.empty((T, self.P, self.C), dtype=torch.bfloat16, device="cuda")
        y = torch.empty((T, self.O), device="cuda")
        minw.minw_group_norm(x.view(T, self.P, self.C), gamma, beta, self.G, EPS, a, act=minw.ACT_HARDTANH,
                             workspace=self._bytes(minw.minw_group_norm_workspace_bytes(T, self.P, self.C, self.G)))
        minw.minw_w4_matvec(a.view(T, self.K), self.codes, self.scales, self.w4_group, y, shift=bias)
        return y


def synthetic(B, H, W, C, classes, seed):
    """Feature maps of `classes` kinds (a pattern each, noise, a scale and an offset of every map's own) and their kinds."""
    g = torch.Generator(device="cuda").manual_seed(0x5EED)         # a stream that no Head draws its weights from
    kinds = torch.randn((classes, H, W, C), generator=g, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    labels = torch.randint(0, classes, (B,), generator=g, device="cuda")
    noise = torch.randn((B, H, W, C), generator=g, device="cuda")
    own = torch.rand((B, 1, 1, 2), generator=g, device="cuda")
    return (kinds[labels] + 2 * noise) * (0.5 + own[..., :1]) + 4 * own[..., 1:], labels


def main():
    head = Head(8, 8, 128, 100)
    for k in range(40):
        loss = head.step(*synthetic(256, 8, 8, 128, 100, 2 + k))
        if k % 10 == 9:
            print(f"step {k + 1}: loss {float(loss):.4f}, gradient norm {float(head.norm):.4f}")
    head.pack()
    x, labels = synthetic(64, 8, 8, 128, 100, 1000)
    packed = torch.cat([head.answer(x[i:i + 1]) for i in range(64)])
    print(f"64 inputs one at a time from {head.codes.numel() / 1e3:.0f} KB of codes: "
          f"{int((packed.argmax(1) == labels).sum())} of 64 right")


if __name__ == "__main__":
    main()
