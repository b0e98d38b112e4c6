"""Operators that adapt a head to many users and serve them at once, as cases
that can be timed and compared: orthogonalised updates of lists of matrices
(Newton-Schulz products), and low-rank adapters of many requests beside a
shared projection (forward, beside 4-bit weights, backward).

A case is a dict of plain values; its "kind" names the operator.  Sizes are
those of the library's configurations (the CIFAR ConvNet's and the heads'
layers) and generic ones.  `run` is the plain form in elementary fp32 torch
operations, or, where `own` is set, the calls a user makes of the library.

`work` counts what an operator cannot do without: each input read once, each
output written once, the products of the cheaper of the two ways to write the
polynomial with symmetric products at half.
"""
import math

import torch

own = False

ACTS = {"none": 0, "hardtanh": 1, "relu": 2, "silu": 3}
ABC = (3.4445, -4.7750, 2.0315)
LR, MU = 2e-2, 0.95

CONVNET = "128x27 128x1152 256x1152 256x2304 512x2304 512x4608 1024x8192 1024x1024 10x1024"
ADAPTERS16 = " ".join(["16x8192 16x1024"] * 8)


def listed():
    return [
        # the gradient of a classifier's weights, ten classes (latency)
        dict(name="orth_classifier", kind="orth", shapes="10x1024", g="bf16", out="bf16"),
        # one large square matrix of bf16 gradients (largest)
        dict(name="orth_large_bf16", kind="orth", shapes="4096x4096", g="bf16", out="bf16"),
        # the step of eight users' adapters (rank 16 beside the ConvNet's first fully connected layer)
        dict(name="step_adapters", kind="step", shapes=ADAPTERS16, g="fp32", w="fp32", nesterov=1),
        # the step of the widest layer of the CIFAR ConvNet
        dict(name="step_fc", kind="step", shapes="1024x8192", g="fp32", w="fp32", nesterov=1),
        # the step of the whole ConvNet: every layer's matrix in one list, tall, wide and ragged ones
        dict(name="step_convnet", kind="step", shapes=CONVNET + " 1001x333 2304x130", g="bf16", w="fp32", nesterov=0),
        # one request through its adapter (latency), the base product at hand
        dict(name="adapt_one", kind="adapt", T=1, K=8192, O=1024, r=16, n=64, run=1, x="bf16", p="bf16", base="fp32",
             y="fp32", act="hardtanh", h=0),
        # a ragged batch in training: fp32 adapters, odd sizes, the inner products kept for the backward
        dict(name="adapt_ragged_fp32", kind="adapt", T=77, K=1155, O=1001, r=12, n=5, run=3, x="fp32", p="fp32",
             base="fp32", y="fp32", act="none", h=1),
        # long prompts of eight users
        dict(name="adapt_long", kind="adapt", T=4096, K=4096, O=4096, r=64, n=8, run=300, x="bf16", p="bf16",
             base="bf16", y="bf16", act="none", h=0),
        # a few users' requests, one input each, through a layer of 4-bit weights and their adapters
        dict(name="w4_adapt_few", kind="w4adapt", T=6, K=8192, O=1024, r=16, n=100, run=1, group=128, x="bf16",
             p="bf16", y="fp32", act="none"),
        # more requests, a larger projection
        dict(name="w4_adapt_many", kind="w4adapt", T=32, K=8192, O=8192, r=32, n=200, run=1, group=64, x="bf16",
             p="bf16", y="bf16", act="silu"),
        # the backward of a ragged batch over fp32 adapters
        dict(name="bwd_ragged_fp32", kind="bwd", T=256, K=8192, O=1001, r=16, n=9, run=7, x="fp32", p="fp32", y="fp32"),
        # ... of long bf16 batches
        dict(name="bwd_long_bf16", kind="bwd", T=2048, K=4096, O=4096, r=32, n=6, run=150, x="bf16", p="bf16", y="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _flops(m, n):
    m, n = min(m, n), max(m, n)
    return min(5 * (3 * m * m * n + m ** 3), 3 * m * m * n + 17 * m ** 3)


def draw(rng):
    kind = rng.choice(["orth", "step", "step", "adapt", "adapt", "w4adapt", "bwd", "bwd"])
    if kind in ("orth", "step"):
        while True:
            shapes = []
            for _ in range(_log(rng, 1, 12)):
                m = _log(rng, 4, 2200)
                n = m * _log(rng, 1, 12) + rng.randint(0, 40)
                shapes.append((m, n) if rng.random() < 0.7 else (n, m))
            if sum(_flops(*s) for s in shapes) <= 6e11 and sum(m * n for m, n in shapes) <= 40_000_000:
                break
        c = dict(kind=kind, shapes=" ".join("%dx%d" % s for s in shapes), g=rng.choice(["bf16", "fp32"]))
        if kind == "orth":
            c["out"] = rng.choice(["bf16", "fp32"])
        else:
            c["w"], c["nesterov"] = rng.choice(["fp32", "fp32", "bf16"]), rng.randint(0, 1)
        return c
    while True:
        c = dict(kind=kind, T=_log(rng, 1, 48 if kind == "w4adapt" else 4096), K=_log(rng, 32, 8192),
                 O=_log(rng, 10, 8192), r=rng.choice([1, 4, 8, 8, 12, 16, 16, 32, 64]), n=_log(rng, 1, 256),
                 run=_log(rng, 1, 400))
        if c["T"] * c["n"] * c["r"] * (c["K"] + c["O"]) <= 1.5e10 and c["T"] * (c["K"] + c["O"]) <= 33_000_000 and \
                c["n"] * c["r"] * (c["K"] + c["O"]) <= 60_000_000:
            break
    c["x"], c["p"], c["y"] = (rng.choice(["bf16", "fp32"]) for _ in range(3))
    if kind == "w4adapt":
        c["group"], c["act"] = rng.choice([32, 64, 128]), rng.choice(list(ACTS))
    if kind == "adapt":
        c["base"], c["act"], c["h"] = rng.choice(["fp32", "bf16", "none"]), rng.choice(list(ACTS)), rng.randint(0, 1)
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4, "none": 0}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _uniform(g, lo, hi, *shape):
    return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo


def _shapes(c):
    return [tuple(int(v) for v in s.split("x")) for s in c["shapes"].split()]


def _gradient(g, m, n):
    """A gradient as a batch of 256 makes it: outer products of errors and activations, some directions a hundred times
    stronger than others, and noise below them."""
    b = 256
    strong = torch.logspace(0, -2, b, device="cuda")
    out = (_normal(g, m, b) * strong) @ torch.relu(_normal(g, b, n)) / 16
    return out.add_(_normal(g, m, n), alpha=0.02).mul_(1e-3)


def _users(g, T, n, run):
    """User of each row: runs of rows of one user, one row in sixteen of none."""
    runs = torch.randint(0, n, (T,), generator=g, device="cuda")
    at = torch.cumsum(torch.rand(T, generator=g, device="cuda") < 1 / run, 0)
    ids = runs[at.clamp_max(T - 1)]
    return torch.where(torch.rand(T, generator=g, device="cuda") < 1 / 16, -1, ids).to(torch.int32)


def prepare(c, seed):
    g = _gen(seed)
    kind = c["kind"]
    if kind in ("orth", "step"):
        shapes = _shapes(c)
        s = dict(c=c, g=[_gradient(g, m, n).to(DT[c["g"]]) for m, n in shapes])
        if kind == "step":
            s["m"] = [_gradient(g, m, n).mul_(3) for m, n in shapes]
            s["w"] = [(_normal(g, m, n) / math.sqrt(n)).clamp_(-1, 1).to(DT[c["w"]]) for m, n in shapes]
        if own:
            from paper_2003_04296_gb300 import minw
            s["gl"] = minw.MatrixList(s["g"])
            if kind == "orth":
                s["out"] = [torch.empty(m, n, dtype=DT[c["out"]], device="cuda") for m, n in shapes]
                s["ol"] = minw.MatrixList(s["out"])
            else:
                s["ml"], s["wl"] = minw.MatrixList(s["m"]), minw.MatrixList(s["w"], limits=1.0)
            s["ws"] = torch.empty(minw.minw_orthogonal_workspace_bytes(s["gl"]), dtype=torch.uint8, device="cuda")
        return s
    T, K, O, r, n = c["T"], c["K"], c["O"], c["r"], c["n"]
    p, y = DT[c["p"]], DT[c["y"]]
    s = dict(c=c, x=_normal(g, T, K).to(DT[c["x"]]), ids=_users(g, T, n, c["run"]),
             down=(_normal(g, n, r, K) / math.sqrt(K)).to(p), up=(_normal(g, n, r, O) * (0.5 / math.sqrt(r))).to(p),
             alpha=_uniform(g, 0.5, 2.0, n))
    if kind == "bwd":
        s["dy"] = (0.1 * _normal(g, T, O)).to(y)
        s["h"] = _chosen(s["x"].float() @ s["down"].float().flatten(0, 1).T, s["ids"], n).sum(1)
    else:
        s["scale"], s["shift"] = _uniform(g, 0.5, 1.5, O), 0.1 * _normal(g, O)
        if kind == "w4adapt":
            u = (_normal(g, O, K) * 2.6).round_().clamp_(-8, 7).add_(8).to(torch.uint8)
            s["codes"] = _pack(u)
            s["scales"] = (_uniform(g, 0.3, 1.7, O, -(-K // c["group"])) / (2.6 * math.sqrt(K))).bfloat16()
        elif c["base"] != "none":
            s["base"] = _normal(g, T, O).to(DT[c["base"]])
    if own:
        from paper_2003_04296_gb300 import minw
        s["ws"] = torch.empty(minw.minw_adapters_workspace_bytes(T, K, O, n, r, kind == "bwd"), dtype=torch.uint8,
                              device="cuda")
        if kind == "bwd":
            s["dx"] = torch.empty_like(s["x"])
            s["ddown"], s["dup"] = torch.empty((n, r, K), device="cuda"), torch.empty((n, r, O), device="cuda")
        else:
            s["y"] = torch.empty((T, O), dtype=y, device="cuda")
            s["h"] = torch.empty((T, r), device="cuda") if c.get("h") else None
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

def _chosen(v, ids, n):
    """v [T][n r] with every user's values -> [T][n][r], zero but for the row's own."""
    mine = torch.arange(n, device=v.device) == ids[:, None]
    return v.view(v.shape[0], n, -1) * mine[:, :, None]


def _act(z, act):
    if act == "hardtanh":
        return z.clamp(-1, 1)
    if act == "relu":
        return z.clamp_min(0)
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _orthogonal(x):
    a, b, c = ABC
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / x.norm().clamp_min(1e-30)
    for _ in range(5):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_2003_04296_gb300 import minw
    c = s["c"]
    kind = c["kind"]
    if kind == "orth":
        minw.minw_orthogonalize(s["gl"], s["ol"], s["ws"])
        return s["out"]
    if kind == "step":
        minw.minw_sgd_orthogonal(s["wl"], s["ml"], s["gl"], LR, s["ws"], momentum=MU, nesterov=bool(c["nesterov"]))
        return s["w"], s["m"]
    if kind == "bwd":
        minw.minw_adapters_backward(s["x"], s["ids"], s["down"], s["up"], s["h"], s["dy"], ddown=s["ddown"],
                                    dup=s["dup"], dx=s["dx"], alpha=s["alpha"], workspace=s["ws"])
        return s["dx"], s["ddown"], s["dup"]
    if kind == "w4adapt":
        minw.minw_w4_adapters(s["x"], s["codes"], s["scales"], c["group"], s["ids"], s["down"], s["up"], s["y"],
                              alpha=s["alpha"], scale=s["scale"], shift=s["shift"], act=ACTS[c["act"]],
                              workspace=s["ws"])
        return s["y"]
    minw.minw_adapters(s["x"], s["ids"], s["down"], s["up"], s["y"], alpha=s["alpha"], base=s.get("base"),
                       scale=s["scale"], shift=s["shift"], act=ACTS[c["act"]], h=s["h"], workspace=s["ws"])
    return (s["y"], s["h"]) if c["h"] else (s["y"],)


def _plain(s):
    c = s["c"]
    kind = c["kind"]
    if kind == "orth":
        return [_orthogonal(g.float()).to(DT[c["out"]]) for g in s["g"]]
    if kind == "step":
        for w, m, g in zip(s["w"], s["m"], s["g"]):
            g = g.float()
            m.mul_(MU).add_(g)
            o = _orthogonal(g + MU * m if c["nesterov"] else m)
            rate = LR * math.sqrt(max(1, w.shape[0] / w.shape[1]))
            w.copy_((w.float() - rate * o).clamp(-1, 1))
        return s["w"], s["m"]
    n, ids, x = c["n"], s["ids"], s["x"].float()
    down, up = s["down"].float().flatten(0, 1), s["up"].float().flatten(0, 1)         # [n r][K], [n r][O]
    alpha = s["alpha"][None, :, None]
    if kind == "bwd":
        dy = s["dy"].float()
        v = (_chosen(dy @ up.T, ids, n) * alpha).flatten(1)
        h = ((torch.arange(n, device=x.device) == ids[:, None])[:, :, None] * s["h"][:, None, :] * alpha).flatten(1)
        return (v @ down).to(DT[c["x"]]), (v.T @ x).view(s["down"].shape), (h.T @ dy).view(s["up"].shape)
    h = _chosen(x @ down.T, ids, n)
    z = (h * alpha).flatten(1) @ up
    if kind == "w4adapt":
        w = _levels(s["codes"], c["K"]).float() - 8
        z = z + x @ (w * s["scales"].float().repeat_interleave(c["group"], dim=1)[:, :c["K"]]).T
    elif c["base"] != "none":
        z = z + s["base"].float()
    y = _act(z * s["scale"] + s["shift"], c["act"]).to(DT[c["y"]])
    return (y, h.sum(1)) if c.get("h") else ((y,) if kind == "adapt" else y)


def exact(c, seed):
    """The operators' definitions in 64 bits on the same inputs."""
    s = prepare(c, seed)
    kind = c["kind"]
    if kind in ("orth", "step"):
        a, b, q = ABC
        outs, ms = [], []
        for k, g in enumerate(s["g"]):
            u = g.double()
            if kind == "step":
                ms.append(MU * s["m"][k].double() + u)
                u = u + MU * ms[k] if c["nesterov"] else ms[k]
            x = u / torch.sqrt((u * u).sum())
            wide = x.shape[0] <= x.shape[1]
            for _ in range(5):
                # a x + b (x x^T) x + q (x x^T)^2 x, from the shorter side
                gx = (x @ x.T) @ x if wide else x @ (x.T @ x)
                ggx = (x @ x.T) @ gx if wide else gx @ (x.T @ x)
                x = a * x + b * gx + q * ggx
            if kind == "step":
                x = torch.clamp(s["w"][k].double() - LR * max(1.0, x.shape[0] / x.shape[1]) ** 0.5 * x, -1, 1)
            outs.append(x)
        return outs if kind == "orth" else (outs, ms)
    x, K, O = s["x"].double(), c["K"], c["O"]
    h = torch.zeros(c["T"], c["r"], dtype=torch.float64, device="cuda")
    if kind == "bwd":
        dy = s["dy"].double()
        dx = torch.zeros_like(x)
        ddown = torch.zeros(c["n"], c["r"], K, dtype=torch.float64, device="cuda")
        dup = torch.zeros(c["n"], c["r"], O, dtype=torch.float64, device="cuda")
        for i in range(c["n"]):
            rows = torch.nonzero(s["ids"] == i).flatten()
            al = float(s["alpha"][i])
            v = al * (dy[rows] @ s["up"][i].double().T)
            dx[rows] = v @ s["down"][i].double()
            ddown[i] = v.T @ x[rows]
            dup[i] = al * (s["h"][rows].double().T @ dy[rows])
        return dx, ddown, dup
    z = torch.zeros(c["T"], O, dtype=torch.float64, device="cuda")
    for i in range(c["n"]):
        rows = torch.nonzero(s["ids"] == i).flatten()
        h[rows] = x[rows] @ s["down"][i].double().T
        z[rows] = float(s["alpha"][i]) * (h[rows] @ s["up"][i].double())
    if kind == "w4adapt":
        for at in range(0, O, 2048):                 # rows of the weights, 2048 at a time
            lv = _levels(s["codes"][at:at + 2048], K).double() - 8
            w = lv * s["scales"][at:at + 2048].repeat_interleave(c["group"], dim=1)[:, :K]
            z[:, at:at + 2048] += x @ w.T
    elif c["base"] != "none":
        z += s["base"].double()
    z = z * s["scale"].double() + s["shift"].double()
    if c["act"] == "hardtanh":
        z = torch.minimum(torch.maximum(z, -torch.ones_like(z)), torch.ones_like(z))
    elif c["act"] == "relu":
        z = torch.maximum(z, torch.zeros_like(z))
    elif c["act"] == "silu":
        z = z * torch.sigmoid(z)
    return (z, h) if c.get("h") else ((z,) if kind == "adapt" else z)


def work(c):
    kind = c["kind"]
    if kind in ("orth", "step"):
        each = SIZE[c["g"]] + (SIZE[c["out"]] if kind == "orth" else 8 + 2 * SIZE[c["w"]])
        return dict(bytes=sum(m * n for m, n in _shapes(c)) * each, flops=sum(_flops(*s) for s in _shapes(c)))
    T, K, O, r, n = c["T"], c["K"], c["O"], c["r"], c["n"]
    users = n * (1 - (1 - 1 / n) ** max(1.0, T / c["run"]))                  # about so many users have rows
    pools = users * r * (K + O) * SIZE[c["p"]]
    if kind == "bwd":
        return dict(bytes=int(pools + n * r * (K + O) * 4 + T * (2 * K * SIZE[c["x"]] + O * SIZE[c["y"]] + r * 4)),
                    flops=4 * T * r * (K + O))
    bytes_ = pools + T * (K * SIZE[c["x"]] + O * (SIZE[c["y"]] + SIZE[c.get("base", "none")]) + 4)
    flops = 2 * T * r * (K + O)
    if kind == "w4adapt":
        bytes_ += O * (-(-K // 2) + 2 * -(-K // c["group"]) + 8)
        flops += 2 * T * O * K
    return dict(bytes=int(bytes_), flops=flops)
