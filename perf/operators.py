"""The operators of a head that is trained in small batches and served one
input at a time, as cases that can be timed and compared: group norm with an
activation on channels-last rows (forward, backward), the global norm of many
gradients with clipping and the clipped update, and products of a few vectors
with 4-bit weights and group scales.

A case is a dict of plain values; its "kind" names the operator.  Sizes are
those of the library's configurations (the CIFAR ConvNet's and ResNet-18's
feature maps and layers, the narrow weight-only networks) and generic ones.
`run` is the plain form in elementary fp32 torch operations, or, where `own`
is set, the calls a user makes of the library.

`work` counts what an operator cannot do without: each input read once, each
output written once.
"""
import math

import torch

own = False

ACTS = {"none": 0, "hardtanh": 1, "relu": 2, "silu": 3}
EPS, LR = 1e-5, 1e-2


def listed():
    return [
        # one small feature map before a classifier: a single image's latency
        dict(name="gn_one_image", kind="gn", B=1, P=64, C=512, G=32, ld=512, x="bf16", y="bf16", act="silu", train=0),
        # first block of the CIFAR ConvNet at its batch: fp32 convolution output to the next layer's bf16 operand
        dict(name="gn_cifar_fp32_to_bf16", kind="gn", B=256, P=1024, C=128, G=32, ld=128, x="fp32", y="bf16",
             act="hardtanh", train=1),
        # images too large for the chip's shared memory, rows wider than the channels read (a feature buffer)
        dict(name="gn_large_rows", kind="gn", B=2, P=501 * 503, C=96, G=8, ld=160, x="bf16", y="bf16", act="silu",
             train=1),
        # backward of a ragged layer: odd batch and pixels, groups of 11 channels that no vector divides
        dict(name="gn_bwd_ragged", kind="gn_bwd", B=37, P=27 * 29, C=132, G=12, ld=132, x="fp32", y="fp32",
             act="hardtanh"),
        # backward of ResNet-18's first stage at its batch (channels 64, 56 x 56)
        dict(name="gn_bwd_stage1", kind="gn_bwd", B=128, P=3136, C=64, G=16, ld=64, x="bf16", y="bf16", act="silu"),
        # the clipped update of a small head's few tensors (latency)
        dict(name="update_small_head", kind="update", tensors=6, values=41_000, g="fp32", w="fp32"),
        # the clipped update of the CIFAR ConvNet: 14 M values in a few large tensors and many vectors
        dict(name="update_convnet", kind="update", tensors=33, values=14_000_000, g="fp32", w="fp32"),
        # clipping the gradients of a deep narrow network: hundreds of small tensors, odd lengths and offsets
        dict(name="clip_narrow_net", kind="clip", tensors=331, values=1_730_000, g="fp32", w="fp32"),
        # the norm and clipping of a large model's bf16 gradients (largest)
        dict(name="clip_large_bf16", kind="clip", tensors=290, values=250_000_000, g="bf16", w="bf16"),
        # one image through the widest fully connected layer of the CIFAR ConvNet
        dict(name="w4_fc_one", kind="w4", T=1, O=1024, K=8192, group=128, x="bf16", y="fp32", act="hardtanh"),
        # a few fp32 vectors, lengths that no tile divides, the finest groups
        dict(name="w4_ragged_fp32", kind="w4", T=5, O=4001, K=4097, group=32, x="fp32", y="fp32", act="none"),
        # a large projection for one token
        dict(name="w4_large_one", kind="w4", T=1, O=16384, K=16384, group=128, x="bf16", y="bf16", act="none"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["gn", "gn", "gn_bwd", "gn_bwd", "update", "clip", "w4", "w4"])
    if kind in ("gn", "gn_bwd"):
        while True:
            G = rng.choice([1, 2, 4, 8, 8, 12, 16, 32, 32])
            C = G * rng.choice([1, 2, 3, 4, 4, 8, 8, 11, 12, 16, 16, 32])
            side = _log(rng, 1, 400)
            P = side * (side if rng.random() < 0.5 else max(1, side + rng.randint(-3, 3)))
            c = dict(kind=kind, B=_log(rng, 1, 256), P=P, C=C, G=G, ld=C + rng.choice([0, 0, 0, 8, 5, 64]),
                     x=rng.choice(["bf16", "fp32"]), y=rng.choice(["bf16", "fp32"]), act=rng.choice(list(ACTS)))
            if kind == "gn":
                c["train"] = rng.randint(0, 1)
            if kind == "gn_bwd":
                c["y"] = c["x"]
            if P * (C // G) >= 16 and 4 <= C <= 1024 and c["B"] * P * c["ld"] <= 33_554_432:
                return c
    if kind in ("update", "clip"):
        c = dict(kind=kind, tensors=_log(rng, 1, 700), values=_log(rng, 1000, 120_000_000),
                 g=rng.choice(["bf16", "fp32"]), w="fp32")
        c["tensors"] = min(c["tensors"], c["values"] // 100)
        if kind == "clip":
            c["w"] = c["g"]
        elif c["g"] == "fp32" and c["values"] > 60_000_000:
            c["values"] //= 2
        return c
    return dict(kind=kind, T=_log(rng, 1, 16), O=_log(rng, 10, 16384), K=_log(rng, 64, 16384),
                group=rng.choice([32, 64, 128, 128]), x=rng.choice(["bf16", "fp32"]), y=rng.choice(["bf16", "fp32"]),
                act=rng.choice(list(ACTS)))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _uniform(g, lo, hi, *shape):
    return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo


def _lengths(c):
    """Lengths of a network's tensors that add up to c["values"]: every other one a vector (biases and norm
    parameters, odd lengths), the rest matrices whose sizes grow with depth."""
    n, total = c["tensors"], c["values"]
    vec = [min(17 + 13 * i % 1024, max(1, total // (2 * n))) if i % 2 else 0 for i in range(n)]
    left, shares = total - sum(vec), [0 if i % 2 else 1 + i for i in range(n)]
    out = [v if v else max(1, left * s // sum(shares)) for v, s in zip(vec, shares)]
    out[0] = max(1, out[0] + total - sum(out))
    return out


def _views(flat, lengths):
    """A flat buffer's consecutive pieces, as gradients lie in one: most start off a 16-byte boundary."""
    return list(torch.split(flat, lengths))


def prepare(c, seed):
    g = _gen(seed)
    kind = c["kind"]
    if kind in ("gn", "gn_bwd"):
        B, P, C, G, ld = c["B"], c["P"], c["C"], c["G"], c["ld"]
        buf = _normal(g, B, P, ld).mul_(0.5 + torch.rand(ld, generator=g, device="cuda")).add_(_normal(g, ld))
        s = dict(c=c, x=buf.to(DT[c["x"]])[:, :, :C], gamma=1 + 0.1 * _normal(g, C), beta=0.1 * _normal(g, C))
        if kind == "gn_bwd":
            s["mean"], s["rstd"] = _stats(s["x"].float(), G)
            dy = 0.1 * _normal(g, B, P, C)
            if c["act"] in ("hardtanh", "relu"):
                # the derivative jumps where |z| = 1 (z = 0): values as near to it as rounding reaches carry no gradient
                z = _affine(s["x"].float(), s["mean"], s["rstd"], s["gamma"], s["beta"], G)
                edge = z.abs() - 1 if c["act"] == "hardtanh" else z
                dy.masked_fill_(edge.abs() < 1e-3, 0.0)
            s["dy"] = dy.to(DT[c["y"]])
        if own:
            from paper_2003_04296_gb300 import minw
            s["ws"] = torch.empty(max(1, minw.minw_group_norm_workspace_bytes(B, P, C, G, kind == "gn_bwd")),
                                  dtype=torch.uint8, device="cuda")
            s["out"] = torch.empty((B, P, C), dtype=DT[c["y"] if kind == "gn" else c["x"]], device="cuda")
            stat = (B, G) if kind == "gn" else (C,)
            s["a"], s["b"] = torch.empty(stat, device="cuda"), torch.empty(stat, device="cuda")
        return s
    if kind in ("update", "clip"):
        lengths = _lengths(c)
        n = sum(lengths)
        grad = _normal(g, n).mul_(1e-3).to(DT[c["g"]])
        s = dict(c=c, g=grad, max_norm=0.37e-3 * math.sqrt(n))          # about a third of the norm: the clipping acts
        if kind == "update":
            s["w"] = _uniform(g, -1, 1, n)
        if own:
            from paper_2003_04296_gb300 import minw
            s["norm"] = torch.empty(1, device="cuda")
            s["gl"] = minw.TensorList(_views(grad, lengths))
            if kind == "update":
                s["wl"] = minw.TensorList(_views(s["w"], lengths), limits=1.0)
            else:
                s["out"] = torch.empty_like(grad)
                s["ol"] = minw.TensorList(_views(s["out"], lengths))
            s["ws"] = torch.empty(minw.minw_grad_workspace_bytes(len(lengths)), dtype=torch.uint8, device="cuda")
        return s
    T, O, K, group = c["T"], c["O"], c["K"], c["group"]
    u = (_normal(g, O, K) * 2.6).round_().clamp_(-8, 7).add_(8).to(torch.uint8)
    s = dict(c=c, codes=_pack(u), scales=(0.02 * _uniform(g, 0.3, 1.7, O, -(-K // group))).bfloat16(),
             x=_normal(g, T, K).to(DT[c["x"]]), scale=_uniform(g, 0.5, 1.5, O), shift=0.1 * _normal(g, O))
    if own:
        s["out"] = torch.empty((T, O), dtype=DT[c["y"]], device="cuda")
    return s


# The 4-bit layout: per row, blocks of 128 values as 16 little-endian 32-bit words; word 4 t + j holds values
# 32 j + 8 t .. + 7 of the block, value i of them in nibble i / 2 + 4 (i % 2), each as its level + 8.
NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]


def _pack(u):
    O, K = u.shape
    p = torch.full((O, -(-K // 128) * 128), 8, dtype=torch.uint8, device=u.device)
    p[:, :K] = u
    p = p.view(O, -1, 4, 4, 8).transpose(2, 3)[..., [0, 2, 4, 6, 1, 3, 5, 7]]        # [O][block][t][j][nibble]
    return (p[..., 0::2] | (p[..., 1::2] << 4)).reshape(O, -1).contiguous()


def _levels(codes, K):
    b = codes.view(codes.shape[0], -1, 4, 4, 4)
    n = torch.stack((b & 15, b >> 4), dim=-1).flatten(-2)[..., NIBBLE]
    return n.transpose(2, 3).reshape(codes.shape[0], -1)[:, :K]


# ---------------------------------------------------------------------------
# the plain forms, and the library's calls
# ---------------------------------------------------------------------------

def _stats(x, G):
    v = x.unflatten(2, (G, -1))
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, (var + EPS).rsqrt()


def _affine(x, mean, rstd, gamma, beta, G):
    xh = (x.unflatten(2, (G, -1)) - mean[:, None, :, None]) * rstd[:, None, :, None]
    return xh.flatten(2) * gamma + beta


def _act(z, act):
    if act == "hardtanh":
        return z.clamp(-1, 1)
    if act == "relu":
        return z.clamp_min(0)
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _dact(z, act):
    if act == "hardtanh":
        return (z.abs() <= 1).to(z.dtype)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_2003_04296_gb300 import minw
    c = s["c"]
    kind = c["kind"]
    if kind == "gn":
        keep = (s["a"], s["b"]) if c["train"] else (None, None)
        minw.minw_group_norm(s["x"], s["gamma"], s["beta"], c["G"], EPS, s["out"], act=ACTS[c["act"]], mean=keep[0],
                             rstd=keep[1], workspace=s["ws"])
        return (s["out"],) + keep if c["train"] else (s["out"],)
    if kind == "gn_bwd":
        minw.minw_group_norm_backward(s["x"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], c["G"], s["out"],
                                      dgamma=s["a"], dbeta=s["b"], act=ACTS[c["act"]], workspace=s["ws"])
        return s["out"], s["a"], s["b"]
    if kind == "update":
        minw.minw_sgd_clip_norm(s["wl"], s["gl"], s["max_norm"], LR, s["norm"], s["ws"])
        return s["w"], s["norm"]
    if kind == "clip":
        minw.minw_grad_clip(s["gl"], s["ol"], s["max_norm"], s["norm"], s["ws"])
        return s["out"], s["norm"]
    minw.minw_w4_matvec(s["x"], s["codes"], s["scales"], c["group"], s["out"], scale=s["scale"], shift=s["shift"],
                        act=ACTS[c["act"]])
    return s["out"]


def _plain(s):
    c = s["c"]
    kind = c["kind"]
    if kind in ("gn", "gn_bwd"):
        G, x = c["G"], s["x"].float()
        if kind == "gn":
            mean, rstd = _stats(x, G)
            y = _act(_affine(x, mean, rstd, s["gamma"], s["beta"], G), c["act"]).to(DT[c["y"]])
            return (y, mean, rstd) if c["train"] else (y,)
        r = s["rstd"][:, None, :, None]
        xh = (x.unflatten(2, (G, -1)) - s["mean"][:, None, :, None]) * r
        dz = s["dy"].float() * _dact(xh.flatten(2) * s["gamma"] + s["beta"], c["act"])
        dzx = dz * xh.flatten(2)
        h = (dz * s["gamma"]).unflatten(2, (G, -1))
        s1, s2 = h.mean((1, 3))[:, None, :, None], (h * xh).mean((1, 3))[:, None, :, None]
        dx = (r * (h - s1 - xh * s2)).flatten(2)
        return dx.to(DT[c["x"]]), dzx.sum((0, 1)), dz.sum((0, 1))
    if kind in ("update", "clip"):
        gf = s["g"].float()
        norm = gf.square().sum().sqrt()
        # a norm that is not finite skips the step
        k = torch.where(norm.isfinite(), (s["max_norm"] / norm).clamp_max(1.0), 0.0)
        if kind == "update":
            s["w"].copy_((s["w"] - LR * (k * gf)).clamp(-1, 1))
            return s["w"], norm.reshape(1)
        return torch.where(norm.isfinite(), k * gf, gf).to(DT[c["g"]]), norm.reshape(1)
    x, group = s["x"].float(), c["group"]
    K = x.shape[1]
    w = _levels(s["codes"], K).float() - 8
    w = w * s["scales"].float().repeat_interleave(group, dim=1)[:, :K]
    return _act((x @ w.T) * s["scale"] + s["shift"], c["act"]).to(DT[c["y"]])


def exact(c, seed):
    """The operators' definitions in 64 bits on the same inputs."""
    s = prepare(c, seed)
    kind = c["kind"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and k not in ("ws", "codes")}
    act = {"none": lambda z: z, "hardtanh": lambda z: torch.minimum(torch.maximum(z, -torch.ones_like(z)),
                                                                  torch.ones_like(z)),
           "relu": lambda z: torch.maximum(z, torch.zeros_like(z)), "silu": lambda z: z * torch.sigmoid(z)}[c["act"]] \
        if "act" in c else None
    if kind in ("gn", "gn_bwd"):
        B, P, C, G = c["B"], c["P"], c["C"], c["G"]
        n = P * (C // G)
        # rows of one group's values: [B G][n]
        rows = lambda t: t.reshape(B, P, G, C // G).permute(0, 2, 1, 3).reshape(B * G, n)           # noqa: E731
        back = lambda t: t.reshape(B, G, P, C // G).permute(0, 2, 1, 3).reshape(B, P, C)            # noqa: E731
        x = rows(d["x"])
        if kind == "gn":
            mean = x.sum(1, keepdim=True) / n
            rstd = 1 / torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / n + EPS)
            y = act(back((x - mean) * rstd) * d["gamma"] + d["beta"])
            return (y, mean.reshape(B, G), rstd.reshape(B, G)) if c["train"] else (y,)
        m, r = d["mean"].reshape(-1, 1), d["rstd"].reshape(-1, 1)
        xh = (x - m) * r
        z = (back(xh) * d["gamma"] + d["beta"]).requires_grad_()
        dz, = torch.autograd.grad(act(z), z, d["dy"])
        z = z.detach()
        h = rows(dz * d["gamma"])
        dx = back(r * (h - h.sum(1, keepdim=True) / n - xh * ((h * xh).sum(1, keepdim=True) / n)))
        return dx, (dz * back(xh)).sum((0, 1)), dz.sum((0, 1))
    if kind in ("update", "clip"):
        norm = torch.sqrt(torch.dot(d["g"], d["g"]))
        k = min(1.0, s["max_norm"] / float(norm))
        if kind == "update":
            return torch.clamp(d["w"] - LR * k * d["g"], -1, 1), norm.reshape(1)
        return k * d["g"], norm.reshape(1)
    K, group = c["K"], c["group"]
    out = []
    for at in range(0, c["O"], 2048):                 # rows of the weights, 2048 at a time
        lv = _levels(s["codes"][at:at + 2048], K).double() - 8
        w = lv * d["scales"][at:at + 2048].repeat_interleave(group, dim=1)[:, :K]
        out.append(d["x"] @ w.T)
    return act(torch.cat(out, dim=1) * d["scale"] + d["shift"])


def work(c):
    kind = c["kind"]
    if kind in ("gn", "gn_bwd"):
        n, stats = c["B"] * c["P"] * c["C"], 8 * c["B"] * c["G"]
        if kind == "gn":
            return dict(bytes=n * (SIZE[c["x"]] + SIZE[c["y"]]) + 8 * c["C"] + (stats if c["train"] else 0), flops=9 * n)
        return dict(bytes=n * (2 * SIZE[c["x"]] + SIZE[c["y"]]) + 16 * c["C"] + stats, flops=16 * n)
    if kind in ("update", "clip"):
        n = sum(_lengths(c))
        if kind == "update":
            return dict(bytes=n * (SIZE[c["g"]] + 2 * SIZE[c["w"]]), flops=6 * n)
        return dict(bytes=2 * n * SIZE[c["g"]], flops=3 * n)
    groups = -(-c["K"] // c["group"])
    return dict(bytes=c["O"] * (-(-c["K"] // 2) + 2 * groups + 8) + c["T"] * (c["K"] * SIZE[c["x"]] + c["O"] * SIZE[c["y"]]),
                flops=2 * c["T"] * c["O"] * c["K"])
