"""Timed cases of the channels-last operators: group norm with an activation and its gradient, 8-bit rows,
8-bit matrix products, and the passes between NCHW planes and channels-last tokens.

A case is one of seven kinds:
  "norm"        - group norm with an activation, as a network that answers runs it;
  "backward"    - its gradient alone, from activations that were kept;
  "train"       - its forward and backward pass, the input kept in between as it is or as 8-bit rows;
  "rows"        - activations written as 8-bit rows and read back;
  "pack", "unpack" - NCHW planes to channels-last tokens, and back;
  "linear"      - the product of 8-bit tokens and 8-bit weights (a pointwise layer, a classifier);
  "norm_linear" - group norm that writes 8-bit tokens, and the product that reads them.
Tensors are [images, pixels, channels], or [tokens, channels] where images do not matter.  8-bit rows are int8 values
[rows, pitch], pitch = columns rounded up to 16 and zeros past the last column, with an fp32 scale for each row.

Sizes are those of the framework's workloads (32 .. 1024 channels on 7x7 .. 112x112 planes, at 1 .. 256 images) or generic.
"""
import math

import torch

own = False             # True: the framework's kernels; False: the plain forms below

DEVICE = "cuda"
EPS = 1e-5
ACTS = ("none", "relu", "silu")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, kind, N, P, C, groups, dtype, act, kept="x", cols=0):
    return {"name": name, "kind": kind, "N": N, "P": P, "C": C, "groups": groups, "dtype": dtype, "act": act, "kept": kept,
            "cols": cols}


def _rows(name, rows, cols, dtype):
    return {"name": name, "kind": "rows", "rows": rows, "cols": cols, "dtype": dtype}


def _planes(name, kind, N, C, P, dtype, to):
    return {"name": name, "kind": kind, "N": N, "C": C, "P": P, "dtype": dtype, "to": to}


def _linear(name, M, K, N, to, bias):
    return {"name": name, "kind": "linear", "M": M, "K": K, "N": N, "to": to, "bias": bias}


def listed():
    return [
        # one image's last stage: 100 KB, launch and latency decide
        _norm("norm_7x7", "norm", 1, 49, 512, 32, "f32", "relu"),
        # a batch of large planes: moving the tensor is what there is to do
        _norm("norm_56x56", "norm", 64, 3136, 256, 32, "bf16", "silu"),
        # gradient on sizes that fit no vector: three groups of 20 channels, odd planes, few images
        _norm("backward_ragged", "backward", 5, 1073, 60, 3, "f32", "silu"),
        # one training step's pass with the input kept in 8 bits: a middle stage at a training batch
        _norm("train_28x28_saved8", "train", 256, 784, 128, 32, "bf16", "silu", "rows8"),
        # 8-bit rows written and read back: odd columns, and a serving batch's activations
        _rows("rows_odd", 5365, 333, "f32"),
        _rows("rows_14x14", 50176, 512, "bf16"),
        # between the convolutions' planes and tokens: into a block at the benchmark's batch, and out of a ragged one
        _planes("pack_28x28", "pack", 256, 128, 784, "f32", "bf16"),
        _planes("unpack_ragged", "unpack", 5, 84, 1073, "bf16", "f32"),
        # a single token against a matrix: reading the weights is what there is to do
        _linear("linear_1_token", 1, 4096, 4096, "bf16", True),
        # a classifier over a ragged batch: no dimension is a multiple of a tile
        _linear("linear_ragged", 197, 1280, 1001, "f32", True),
        # many tokens: the largest product
        _linear("linear_8192", 8192, 4096, 8192, "bf16", False),
        # the pointwise layer of a block: normalised, activated, rounded to 8 bits, multiplied
        _norm("norm_linear_14x14", "norm_linear", 64, 196, 512, 32, "bf16", "silu", "x", 1024),
    ]


# ---- drawn cases -------------------------------------------------------------------------------
MAX_ELEMENTS = 51_000_000       # of one tensor, and
MAX_PRODUCT = 270e9             # multiplications: both no more than the largest listed case's


def _spread(rng, low, high):
    """A whole number between low and high, spread over their logarithm."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def _channels(rng, most=64):
    """(channels, groups): usual groups of 4 .. 64 channels, and odd ones."""
    if rng.random() < 0.6:
        return rng.choice([(32, 8), (64, 32), (96, 8), (128, 32), (192, 32), (256, 32), (320, 32), (384, 16), (512, 32), (960, 32),
                           (1024, 32), (1280, 32)])
    groups = rng.choice([1, 2, 3, 4, 6, 8, 16, 32])
    return groups * rng.randint(1, most), groups


def draw(rng):
    kind = rng.choice(["norm", "norm", "backward", "train", "rows", "pack", "unpack", "linear", "linear", "norm_linear"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "rows":
        cols = _spread(rng, 16, 4096)
        case = _rows("", _spread(rng, 1, min(200_000, MAX_ELEMENTS // cols)), cols, dtype)
    elif kind in ("pack", "unpack"):
        C, P = _spread(rng, 3, 1024), _spread(rng, 1, 12544)
        case = _planes("", kind, _spread(rng, 1, max(1, min(256, MAX_ELEMENTS // (C * P)))), C, P, dtype, rng.choice(["f32", "bf16"]))
    elif kind == "linear":
        M, K, N = _spread(rng, 1, 16384), _spread(rng, 16, 8192), _spread(rng, 16, 8192)
        M = max(1, min(M, int(MAX_PRODUCT / (K * N)), MAX_ELEMENTS // max(K, N)))
        case = _linear("", M, K, N, rng.choice(["f32", "bf16"]), rng.random() < 0.5)
    else:
        C, groups = _channels(rng)
        # at least 16 values in a group: what fewer leave of a gradient is what cancellation leaves
        P = _spread(rng, -(-16 * groups // C), 12544)
        N = _spread(rng, 1, max(1, min(256, MAX_ELEMENTS // (C * P) // (2 if kind == "train" else 1))))
        kept = rng.choice(["x", "rows8"]) if kind in ("backward", "train") else "x"
        cols = 0
        if kind == "norm_linear":
            dtype, cols = "bf16", _spread(rng, 16, 2048)
            N = max(1, min(N, MAX_ELEMENTS // (P * cols)))
        # gradients through smooth activations only: ReLU's jumps, and on which side of zero a value within rounding of it
        # lies is not for a comparison to say
        act = rng.choice(("none", "silu") if kind in ("backward", "train") else ACTS)
        case = _norm("", kind, N, P, C, groups, dtype, act, kept, cols)
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, device=DEVICE, generator=g)


def _activations(g, rows, cols):
    """What a convolution leaves: channels with offsets and spreads of their own."""
    return _normal(g, rows, cols).mul_(torch.exp(0.5 * _normal(g, cols))).add_(0.5 * _normal(g, cols))


def _rows8(x):
    """(int8 values [rows, pitch], scales [rows]) of x [rows, cols]: the plain form of writing 8-bit rows."""
    x = x.float()
    big = x.abs().amax(1, keepdim=True)
    top = torch.full_like(big, 127.0)       # tensors by tensors: dividing by a number would multiply by its reciprocal
    up = torch.where(big < 2.0 ** -64, 2.0 ** 64, 1.0)
    inv = top / torch.where(big > 0, big * up, 1.0)
    q = torch.round(x * up * inv)
    return torch.nn.functional.pad(q, (0, -x.shape[1] % 16)).to(torch.int8), (big / top)[:, 0]


def _statistics(x, groups):
    """(mean, 1 / standard deviation) [images, groups, 2] of x [images, pixels, channels]."""
    N, P, C = x.shape
    x = x.float().view(N, P, groups, C // groups)
    mean = x.mean((1, 3), keepdim=True)
    var = (x - mean).square().mean((1, 3))
    return torch.stack((mean[:, 0, :, 0], torch.rsqrt(var + EPS)), 2)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    kind, s = case["kind"], {"case": dict(case)}
    if kind == "rows":
        R, C, t = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"] = _activations(g, R, C).to(t)
        s["q"] = torch.empty(R, -(-C // 16) * 16, dtype=torch.int8, device=DEVICE), torch.empty(R, device=DEVICE)
        s["out"] = torch.empty(R, C, dtype=t, device=DEVICE)
    elif kind in ("pack", "unpack"):
        N, C, P, t = case["N"], case["C"], case["P"], TYPES[case["dtype"]]
        s["x"] = _normal(g, *((N, C, P) if kind == "pack" else (N, P, C))).to(t)
        s["out"] = torch.empty((N, P, C) if kind == "pack" else (N, C, P), dtype=TYPES[case["to"]], device=DEVICE)
    elif kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        s["a"] = _rows8(torch.nn.functional.silu(_activations(g, M, K)))
        s["w"] = _rows8(_normal(g, N, K) * math.sqrt(2.0 / K))
        s["bias"] = 0.1 * _normal(g, N) if case["bias"] else None
        s["out"] = torch.empty(M, N, dtype=TYPES[case["to"]], device=DEVICE)
    else:
        N, P, C, G, t = case["N"], case["P"], case["C"], case["groups"], TYPES[case["dtype"]]
        rows = N * P
        s["x"] = _activations(g, rows, C).to(t).view(N, P, C)
        s["gamma"], s["beta"] = 1 + 0.2 * _normal(g, C), 0.2 * _normal(g, C)
        s["stats"] = torch.empty(N, G, 2, device=DEVICE)
        s["saved"] = torch.empty(rows, -(-C // 16) * 16, dtype=torch.int8, device=DEVICE), torch.empty(rows, device=DEVICE)
        if kind == "norm_linear":
            s["w"] = _rows8(_normal(g, case["cols"], C) * math.sqrt(2.0 / C))
            s["out"] = torch.empty(rows, case["cols"], dtype=t, device=DEVICE)
        else:
            s["y"] = torch.empty_like(s["x"])
        if kind in ("backward", "train"):
            s["dy"] = (_normal(g, rows, C) * torch.exp(0.3 * _normal(g, C))).to(t).view(N, P, C)
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = torch.empty(C, device=DEVICE), torch.empty(C, device=DEVICE)
        if kind == "backward":
            s["stats"] = _statistics(s["x"], G)
            if case["kept"] == "rows8":
                s["saved"] = _rows8(s["x"].view(rows, C))
    return s


# ---- plain forms: elementary operations in 32 bits, rounded once at the end -----------------------
def _read8(saved, cols):
    q, scale = saved
    return q[:, :cols].float() * scale[:, None]


def _spread_stats(stats, C):
    """stats [images, groups, 2] as (mean, rstd) [images, 1, channels]."""
    each = stats.repeat_interleave(C // stats.shape[1], 1)
    return each[:, None, :, 0], each[:, None, :, 1]


def _activate(z, act):
    return z if act == "none" else z.clamp_min(0) if act == "relu" else z / (1 + torch.exp(-z))


def _slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _forward(x, stats, gamma, beta, act):
    mean, rstd = _spread_stats(stats, x.shape[2])
    return _activate((x - mean) * rstd * gamma + beta, act)


def _backward(dy, x, stats, gamma, beta, groups, act):
    N, P, C = x.shape
    mean, rstd = _spread_stats(stats, C)
    xh = (x - mean) * rstd
    dz = dy * _slope(xh * gamma + beta, act)
    dbeta, dgamma = dz.sum((0, 1)), (dz * xh).sum((0, 1))
    t = dz * gamma
    m = P * (C // groups)
    a = t.view(N, P, groups, -1).sum((1, 3)) / m
    b = (t * xh).view(N, P, groups, -1).sum((1, 3)) / m
    each = torch.stack((a, b), 2).repeat_interleave(C // groups, 1)[:, None]
    return rstd * (t - each[..., 0] - xh * each[..., 1]), dgamma, dbeta


def _product(a, w, bias):
    out = (a[0].float() @ w[0].float().t()) * a[1][:, None] * w[1]
    return out if bias is None else out + bias


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "rows":
        q, scale = _rows8(s["x"])
        return {"x": _read8((q, scale), c["cols"]).to(s["x"].dtype), "scale": scale}
    if kind in ("pack", "unpack"):
        return s["x"].float().transpose(1, 2).to(TYPES[c["to"]]).contiguous()
    if kind == "linear":
        return _product(s["a"], s["w"], s["bias"]).to(TYPES[c["to"]])
    t, G, C = TYPES[c["dtype"]], c["groups"], c["C"]
    x = s["x"].float()
    if kind == "backward":
        if c["kept"] == "rows8":
            x = _read8(s["saved"], C).view(x.shape)
        dx, dgamma, dbeta = _backward(s["dy"].float(), x, s["stats"], s["gamma"], s["beta"], G, c["act"])
        return {"dx": dx.to(t), "dgamma": dgamma, "dbeta": dbeta}
    stats = _statistics(x, G)
    y = _forward(x, stats, s["gamma"], s["beta"], c["act"])
    if kind == "norm":
        return y.to(t)
    if kind == "norm_linear":
        return _product(_rows8(y.view(-1, C)), s["w"], None).to(t)
    if c["kept"] == "rows8":
        x = _read8(_rows8(x.view(-1, C)), C).view(x.shape)
    dx, dgamma, dbeta = _backward(s["dy"].float(), x, stats, s["gamma"], s["beta"], G, c["act"])
    return {"y": y.to(t), "stats": stats, "dx": dx.to(t), "dgamma": dgamma, "dbeta": dbeta}


# ---- the framework's calls ------------------------------------------------------------------------
def _own(s):
    from paper_2006_09791_amd import binding as b
    c = s["case"]
    kind = c["kind"]
    if kind == "rows":
        b.gspc_quantize_rows(s["x"], out=s["q"])
        return {"x": b.gspc_dequantize_rows(s["q"], c["cols"], out=s["out"]), "scale": s["q"][1]}
    if kind == "pack":
        return b.gspc_pack_channels_last(s["x"], out=s["out"])
    if kind == "unpack":
        return b.gspc_unpack_channels_last(s["x"], out=s["out"])
    if kind == "linear":
        return b.gspc_matmul_i8(s["a"], s["w"], bias=s["bias"], out=s["out"])
    act = {"none": b.ACT_NONE, "relu": b.ACT_RELU, "silu": b.ACT_SILU}[c["act"]]
    gamma, beta, G = s["gamma"], s["beta"], c["groups"]
    if kind == "norm":
        return b.gspc_group_norm(s["x"], gamma, beta, G, EPS, act, out=s["y"])
    if kind == "norm_linear":
        rows8 = b.gspc_group_norm(s["x"], gamma, beta, G, EPS, act, out=s["saved"])
        return b.gspc_matmul_i8(rows8, s["w"], out=s["out"])
    kept = s["saved"] if c["kept"] == "rows8" else s["x"]
    if kind == "train":
        b.gspc_group_norm(s["x"], gamma, beta, G, EPS, act, out=s["y"], stats=s["stats"],
                          saved=s["saved"] if c["kept"] == "rows8" else None)
    b.gspc_group_norm_backward(s["dy"], kept, s["stats"], gamma, beta, G, act, dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    out = {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    return out if kind == "backward" else {"y": s["y"], "stats": s["stats"], **out}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2}
    if kind == "rows":
        R, C, e = case["rows"], case["cols"], size[case["dtype"]]
        return {"bytes": R * (2 * C * e + 2 * (C + 4)), "flops": 5 * R * C}
    if kind in ("pack", "unpack"):
        return {"bytes": case["N"] * case["C"] * case["P"] * (size[case["dtype"]] + size[case["to"]]), "flops": 0}
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": (M + N) * (K + 4) + M * N * size[case["to"]] + (4 * N if case["bias"] else 0), "flops": 2 * M * K * N}
    rows, C, e = case["N"] * case["P"], case["C"], size[case["dtype"]]
    n, each = rows * C, 12 if case["act"] == "silu" else 8
    x = rows * (C + 4) if case["kept"] == "rows8" else n * e
    backward, vectors = n * 2 * e + x, 16 * C + 8 * case["N"] * case["groups"]
    if kind == "norm":
        return {"bytes": 2 * n * e + 8 * C, "flops": each * n}
    if kind == "backward":
        return {"bytes": backward + vectors, "flops": 2 * each * n}
    if kind == "train":
        return {"bytes": 2 * n * e + (x if case["kept"] == "rows8" else 0) + backward + 2 * vectors, "flops": 3 * each * n}
    cols = case["cols"]
    return {"bytes": n * e + 2 * rows * (C + 4) + cols * (C + 4) + rows * cols * e, "flops": (each + 2 * cols) * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_rows8(x):
    top = x.abs().max(1).values[:, None]
    step = top / 127
    return torch.where(top > 0, (x / torch.where(top > 0, step, torch.ones_like(step))).round(), torch.zeros_like(x)) * step, step[:, 0]


def _exact_norm(x, gamma, beta, G, act, stats=None):
    """(x hat, z, mean, rstd), with x as [images, pixels, groups, channels of a group]."""
    N, P, C = x.shape
    x = x.reshape(N, P, G, C // G)
    if stats is None:
        count = P * (C // G)
        mean = x.sum(dim=(1, 3)) / count
        rstd = 1 / ((x - mean[:, None, :, None]).pow(2).sum(dim=(1, 3)) / count + EPS).sqrt()
    else:
        mean, rstd = stats[..., 0], stats[..., 1]
    xh = (x - mean[:, None, :, None]) * rstd[:, None, :, None]
    return xh, xh * gamma.reshape(G, -1) + beta.reshape(G, -1), mean, rstd


def _exact_act(z, act):
    return {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)), "silu": lambda: z * torch.sigmoid(z)}[act]()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    up = lambda k: s[k].double()  # noqa: E731
    if kind == "rows":
        x, scale = _exact_rows8(up("x"))
        return {"x": x, "scale": scale}
    if kind in ("pack", "unpack"):
        return up("x").permute(0, 2, 1).contiguous()
    if kind == "linear":
        a, w = (s[k][0].double() * s[k][1].double()[:, None] for k in ("a", "w"))
        y = torch.matmul(a, w.T.contiguous())
        return y if s["bias"] is None else y + up("bias")
    G, act, shape = case["groups"], case["act"], s["x"].shape
    gamma, beta, x = up("gamma"), up("beta"), up("x")
    rows = x.reshape(-1, shape[2])
    if kind == "backward":
        stats = up("stats")
        if case["kept"] == "rows8":
            x = (s["saved"][0].double() * s["saved"][1].double()[:, None])[:, :shape[2]].reshape(shape)
    else:
        _, z, mean, rstd = _exact_norm(x, gamma, beta, G, act)
        y = _exact_act(z, act).reshape(shape)
        if kind == "norm":
            return y
        if kind == "norm_linear":
            w = (s["w"][0].double() * s["w"][1].double()[:, None])[:, :shape[2]]
            return torch.matmul(_exact_rows8(y.reshape(rows.shape))[0], w.T.contiguous())
        stats = torch.stack((mean, rstd), -1)
        if case["kept"] == "rows8":
            x = _exact_rows8(rows)[0].reshape(shape)
    xh, z, _, rstd = _exact_norm(x, gamma, beta, G, act, stats)
    sig = torch.sigmoid(z)
    slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": sig + z * sig * (1 - sig)}[act]
    dz = up("dy").reshape(xh.shape) * slope
    dgamma, dbeta = (dz * xh).sum(dim=(0, 1)).reshape(-1), dz.sum(dim=(0, 1)).reshape(-1)
    dxh = dz * gamma.reshape(G, -1)
    count = xh.shape[1] * xh.shape[3]
    centre = dxh.sum(dim=(1, 3), keepdim=True) / count
    along = (dxh * xh).sum(dim=(1, 3), keepdim=True) / count
    dx = ((dxh - centre - xh * along) * rstd[:, None, :, None]).reshape(shape)
    out = {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    return out if kind == "backward" else {"y": y, "stats": stats, **out}
