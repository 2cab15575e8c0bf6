"""Timed cases of the residual block's operators on tokens: 8-bit float rows and their products with their gradients, norms before and
after a block fused with its gate and residual scale, and dropout whose mask is never stored.

A case is one of seven kinds:
  "rows"    - values written as 8-bit float rows along both directions, and both read back;
  "linear"  - the product of 8-bit float tokens and weights (a pointwise layer, a classifier);
  "step"    - a pointwise layer's training pass: its output and both of its gradients, all three products in 8 bits;
  "join"    - a block's output normalised, gated and added to the residual stream, and the stream normalised for the next block;
  "train"   - that and its gradient, with dropout, the gradient from a stream and statistics that were kept;
  "block"   - a residual block as a network that answers runs it: norm and activation written in 8 bits, product, join;
  "dropout" - dropout of a tensor and of the gradient behind it.

8-bit float rows are e4m3 values [rows, pitch], pitch = columns rounded up to 128 and zeros past the last column, with a byte for
each 128 columns [rows, pitch / 128 rounded up to 4]: the exponent, plus 127, of the power of two that they are multiplied by.

Dropout's random numbers are Philox 4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) of the counter
(column / 8, row, low and high word of the call's number) under the seed as key: eight 16-bit numbers for eight columns.

Sizes are those of the framework's workloads (32 .. 1024 channels on 7x7 .. 112x112 planes, at 1 .. 256 images) or generic.
"""
import math

import torch

own = False             # True: the framework's kernels; False: the plain forms below

DEVICE = "cuda"
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rows(name, rows, cols, dtype):
    return {"name": name, "kind": "rows", "rows": rows, "cols": cols, "dtype": dtype}


def _linear(name, M, K, N, to, bias):
    return {"name": name, "kind": "linear", "M": M, "K": K, "N": N, "to": to, "bias": bias}


def _step(name, M, K, N):
    return {"name": name, "kind": "step", "M": M, "K": K, "N": N}


def _join(name, kind, N, P, C, dtype, post, pre, gate, act, scale, drop):
    return {"name": name, "kind": kind, "N": N, "P": P, "C": C, "dtype": dtype, "post": post, "pre": pre, "gate": gate, "act": act,
            "scale": scale, "drop": drop}


def _dropout(name, rows, cols, dtype, drop):
    return {"name": name, "kind": "dropout", "rows": rows, "cols": cols, "dtype": dtype, "drop": drop}


def listed():
    return [
        # weights and activations on sizes that fit no tile, and a stage's activations for a training step's two directions
        _rows("rows_odd", 5365, 333, "f32"),
        _rows("rows_28x28", 50176, 512, "bf16"),
        # a single token against a matrix: reading the weights is what there is to do
        _linear("linear_1_token", 1, 4096, 4096, "bf16", True),
        # a classifier over a ragged batch: no dimension is a multiple of a tile
        _linear("linear_ragged", 197, 1280, 1001, "f32", True),
        # many tokens: the largest product
        _linear("linear_8192", 8192, 4096, 8192, "bf16", False),
        # a training batch's pointwise layer in the last stage but one: the gradient of the weights sums over all tokens
        _step("step_14x14", 12544, 512, 1024),
        # one token between two blocks: launch and latency decide
        _join("join_1_token", "join", 1, 1, 4096, "bf16", "rms", "rms", "none", "none", 1.0, 0.0),
        # a training step between two blocks: a middle stage at a training batch
        _join("train_28x28", "train", 64, 784, 512, "bf16", "layer", "layer", "channel", "silu", 1.0, 0.1),
        # few images of odd planes, a gate for each image
        _join("train_ragged", "train", 5, 1073, 60, "f32", "rms", "layer", "image", "none", 0.5, 0.25),
        # a residual block of a network that answers
        _join("block_14x14", "block", 64, 196, 512, "bf16", "layer", "layer", "channel", "silu", 1.0, 0.0),
        # dropout inside a wide residual block, forward and back
        _dropout("dropout_56x56", 200704, 256, "bf16", 0.3),
        _dropout("dropout_odd", 5365, 333, "f32", 0.5),
    ]


# ---- drawn cases -------------------------------------------------------------------------------
MAX_ELEMENTS = 51_000_000       # of one tensor, and
MAX_PRODUCT = 270e9             # multiplications: both no more than the largest listed case's


def _spread(rng, low, high):
    """A whole number between low and high, spread over their logarithm."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["rows", "linear", "linear", "step", "join", "train", "train", "block", "dropout"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("rows", "dropout"):
        cols = _spread(rng, 16, 4096)
        rows = _spread(rng, 1, min(200_000, MAX_ELEMENTS // 2 // cols))
        case = _rows("", rows, cols, dtype) if kind == "rows" else _dropout("", rows, cols, dtype, rng.choice([0.05, 0.1, 0.3, 0.5, 0.9]))
    elif kind == "linear":
        M, K, N = _spread(rng, 1, 16384), _spread(rng, 16, 8192), _spread(rng, 16, 8192)
        M = max(1, min(M, int(MAX_PRODUCT / (K * N)), MAX_ELEMENTS // max(K, N)))
        case = _linear("", M, K, N, rng.choice(["f32", "bf16"]), rng.random() < 0.5)
    elif kind == "step":
        K, N = _spread(rng, 16, 2048), _spread(rng, 16, 2048)
        case = _step("", _spread(rng, 16, min(65536, MAX_ELEMENTS // 2 // max(K, N))), K, N)
    else:
        C = rng.choice([32, 64, 96, 128, 192, 256, 320, 384, 512, 960, 1024, 1280, 2048]) if rng.random() < 0.5 else _spread(rng, 16, 8192)
        if kind == "block":
            dtype, C = "bf16", min(C, 2048)
        P = _spread(rng, 1, 3136)
        N = _spread(rng, 1, max(1, min(256, MAX_ELEMENTS // 2 // (C * P))))
        drop = rng.choice([0.0, 0.1, 0.25, 0.5]) if kind == "train" else 0.0
        case = _join("", kind, N, P, C, dtype, rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer"]),
                     rng.choice(["none", "channel", "image"]), rng.choice(["none", "silu"]), rng.choice([1.0, 0.5, 0.8]), drop)
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, device=DEVICE, generator=g)


def _activations(g, rows, cols):
    """What a layer leaves: channels with offsets and spreads of their own."""
    return _normal(g, rows, cols).mul_(torch.exp(0.5 * _normal(g, cols))).add_(0.5 * _normal(g, cols))


def _pow2(k):
    """2^k in 32 bits, k from -127 on, by its exponent's bits: the device's exponential may be off by a rounding, its shift is not."""
    return torch.where(k < -126, torch.full((), 2.0 ** -127, device=k.device), (k.clamp_min(-126).int() + 127 << 23).view(torch.float32))


def _float8(x):
    """(e4m3 values, as fp32 [rows, blocks, 128], and exponents [rows, blocks]) of x [rows, cols]."""
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % 128)).view(x.shape[0], -1, 128)
    part, k = torch.frexp(x.abs().amax(2))
    k = torch.where(part > 0, torch.where(part > 0.875, k - 8, k - 9), -127).clamp_min(-127)    # 448 = 0.875 2^9
    x = x * _pow2(-k)[:, :, None]
    e = (torch.frexp(x.abs())[1] - 1).clamp_min(-6) - 3        # neighbours are 2^e apart
    return torch.round(x * _pow2(-e)) * _pow2(e), k


def _store8(x):
    """Such rows as they are kept: (values [rows, pitch], bytes [rows, blocks rounded up to 4])."""
    q, k = _float8(x)
    return (q.view(q.shape[0], -1).to(torch.float8_e4m3fn),
            torch.nn.functional.pad(k + 127, (0, -k.shape[1] % 4)).to(torch.uint8).contiguous())


def _read8(q, k, cols):
    return (q * _pow2(k)[:, :, None]).view(q.shape[0], -1)[:, :cols]


def _load8(pair, cols):
    """The values that stored rows stand for."""
    q, scale = pair
    q = q.float().view(q.shape[0], -1, 128)
    return _read8(q, scale[:, :q.shape[1]].int() - 127, cols)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    kind, s = case["kind"], {"case": dict(case)}
    empty = lambda *shape, t=torch.float32: torch.empty(*shape, dtype=t, device=DEVICE)  # noqa: E731
    rows8 = lambda rows, cols: (empty(rows, -(-cols // 128) * 128, t=torch.float8_e4m3fn),  # noqa: E731
                                empty(rows, -(-cols // 512) * 4, t=torch.uint8))
    if kind == "rows":
        R, C, t = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"] = _activations(g, R, C).to(t)
        s["rows"], s["columns"] = rows8(R, C), rows8(C, R)
        s["out"], s["out_t"] = empty(R, C, t=t), empty(C, R, t=t)
    elif kind == "dropout":
        R, C, t = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"], s["dy"] = _activations(g, R, C).to(t), _normal(g, R, C).to(t)
        s["y"], s["dx"] = empty(R, C, t=t), empty(R, C, t=t)
    elif kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        s["a"] = _store8(torch.nn.functional.silu(_activations(g, M, K)))
        s["w"] = _store8(_normal(g, N, K) * math.sqrt(2.0 / K))
        s["bias"] = 0.1 * _normal(g, N) if case["bias"] else None
        s["out"] = empty(M, N, t=TYPES[case["to"]])
    elif kind == "step":
        M, K, N, t = case["M"], case["K"], case["N"], torch.bfloat16
        s["x"] = torch.nn.functional.silu(_activations(g, M, K)).to(t)
        s["w"] = _normal(g, N, K) * math.sqrt(2.0 / K)                  # the master copy: another one after each step
        s["dy"] = (_normal(g, M, N) * torch.exp(0.3 * _normal(g, N))).to(t)
        for name, rows, cols in (("x8", M, K), ("w8", N, K), ("dy8", M, N)):
            s[name], s[name + "t"] = rows8(rows, cols), rows8(cols, rows)
        s["y"], s["dx"], s["dw"] = empty(M, N, t=t), empty(M, K, t=t), empty(N, K)
    else:
        N, P, C, t = case["N"], case["P"], case["C"], TYPES[case["dtype"]]
        rows = N * P
        s["x"], s["h"] = (_activations(g, rows, C).to(t) for _ in range(2))
        for k in ("post", "pre"):
            s[k + "_gamma"] = 1 + 0.2 * _normal(g, C)
            s[k + "_beta"] = 0.2 * _normal(g, C) if case[k] == "layer" else None
        if case["post"] == "none":
            s["post_gamma"] = s["post_beta"] = None
        s["gate"] = None if case["gate"] == "none" else 0.5 + 0.3 * _normal(g, 1 if case["gate"] == "channel" else N, C)
        s["xo"], s["z"] = empty(rows, C, t=t), empty(rows, C, t=t)
        if kind == "train":
            s["dz"], s["dxo"] = ((_normal(g, rows, C) * torch.exp(0.3 * _normal(g, C))).to(t) for _ in range(2))
            s["stats"] = empty(rows, 4)
            s["dx"], s["dh"] = empty(rows, C, t=t), empty(rows, C, t=t)
            for k in ("gate", "post_gamma", "post_beta", "pre_gamma", "pre_beta"):
                s["d" + k] = None if s[k] is None else torch.empty_like(s[k])
        if kind == "block":
            s["z8"], s["w"] = rows8(rows, C), _store8(_normal(g, C, C) * math.sqrt(2.0 / C))
    # the generator's key, and the number of the call in it
    s["seed"], s["offset"] = (int(torch.randint(1 << 62, (1,), device=DEVICE, generator=g)) for _ in range(2))
    if kind == "train":     # what the forward pass kept: to which side a value between two bf16 numbers was rounded is no matter of the gradient
        xo, _, s["kept_stats"] = _join_plain(s, s["x"].float(), s["h"].float(), _mask_of(s))
        s["kept"] = xo.to(t)
    return s


# ---- plain forms: elementary operations in 32 bits, rounded once at the end -----------------------
WORD = 0xffffffff


def _philox(words, key):
    """Ten rounds over four words of 32 bits, tensors of int64 (products wrap, which their halves do not see)."""
    c0, c1, c2, c3 = words
    k0, k1 = key & WORD, key >> 32 & WORD
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (p1 >> 32 & WORD) ^ c1 ^ k0, p1 & WORD, (p0 >> 32 & WORD) ^ c3 ^ k1, p0 & WORD
        k0, k1 = k0 + 0x9E3779B9 & WORD, k1 + 0xBB67AE85 & WORD
    return c0, c1, c2, c3


def _mask(rows, cols, drop, seed, offset):
    """What dropout multiplies by, [rows, cols]: zero, or what makes up for the dropped."""
    limit = round(drop * 65536)
    number = lambda n: torch.arange(n, dtype=torch.int64, device=DEVICE)  # noqa: E731
    c0, c1 = torch.broadcast_tensors(number(-(-cols // 8)), number(rows)[:, None])
    words = _philox((c0, c1, torch.full_like(c0, offset & WORD), torch.full_like(c0, offset >> 32 & WORD)), seed)
    halves = torch.stack([h for w in words for h in (w & 0xffff, w >> 16)], 2).view(rows, -1)[:, :cols]
    return torch.where(halves >= limit, 65536.0 / (65536 - limit), 0.0)


def _mask_of(s):
    c = s["case"]
    return _mask(c["N"] * c["P"], c["C"], c["drop"], s["seed"], s["offset"]) if c["drop"] else 1.0


def _normalise(x, kind):
    """(x hat, mean, 1 / deviation), the last two [rows, 1]."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    if kind == "none":
        return x, mean, torch.ones_like(mean)
    rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    return (x - mean) * rstd, mean, rstd


def _affine(xh, gamma, beta):
    y = xh if gamma is None else xh * gamma
    return y if beta is None else y + beta


def _each_row(gate, rows):
    return 1.0 if gate is None else gate.repeat_interleave(rows // gate.shape[0], 0) if gate.shape[0] > 1 else gate


def _join_plain(s, x, h, mask):
    """(x', z, statistics)"""
    c = s["case"]
    hh, m1, r1 = _normalise(h, c["post"])
    xo = c["scale"] * x + _each_row(s["gate"], len(x)) * (_affine(hh, s["post_gamma"], s["post_beta"]) * mask)
    xh, m2, r2 = _normalise(xo, c["pre"])
    z = _affine(xh, s["pre_gamma"], s["pre_beta"])
    return xo, z if c["act"] == "none" else z / (1 + torch.exp(-z)), torch.cat((m1, r1, m2, r2), 1)


def _norm_gradient(t, xh, rstd, kind):
    """Through x hat: t is its gradient."""
    if kind == "none":
        return t
    d = t - xh * (t * xh).mean(1, keepdim=True)
    return (d - t.mean(1, keepdim=True) if kind == "layer" else d) * rstd


def _join_gradient(s, xo, h, stats, mask):
    c, rows = s["case"], len(h)
    m1, r1, m2, r2 = stats.split(1, 1)
    xh, hh = (xo - m2) * r2, (h - m1) * r1
    dv = s["dz"].float()
    if c["act"] == "silu":
        v = _affine(xh, s["pre_gamma"], s["pre_beta"])
        sig = 1 / (1 + torch.exp(-v))
        dv = dv * sig * (1 + v * (1 - sig))
    total = s["dxo"].float() + _norm_gradient(dv * s["pre_gamma"], xh, r2, c["pre"])
    du = mask * total * _each_row(s["gate"], rows)
    out = {"dx": c["scale"] * total,
           "dh": _norm_gradient(du if s["post_gamma"] is None else du * s["post_gamma"], hh, r1, c["post"]),
           "dpre_gamma": (dv * xh).sum(0)}
    if s["pre_beta"] is not None:
        out["dpre_beta"] = dv.sum(0)
    if s["gate"] is not None:
        dropped = _affine(hh, s["post_gamma"], s["post_beta"]) * mask
        out["dgate"] = (total * dropped).view(s["gate"].shape[0], -1, h.shape[1]).sum(1)
    if s["post_gamma"] is not None:
        out["dpost_gamma"] = (du * hh).sum(0)
    if s["post_beta"] is not None:
        out["dpost_beta"] = du.sum(0)
    return out


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "rows":
        t, x = s["x"].dtype, s["x"]
        return {"rows": _read8(*_float8(x), c["cols"]).to(t), "columns": _read8(*_float8(x.t()), c["rows"]).to(t)}
    if kind == "dropout":
        mask = _mask(c["rows"], c["cols"], c["drop"], s["seed"], s["offset"])
        return {"y": (s["x"].float() * mask).to(s["x"].dtype), "dx": (s["dy"].float() * mask).to(s["x"].dtype)}
    if kind == "linear":
        out = _load8(s["a"], c["K"]) @ _load8(s["w"], c["K"]).t()
        return (out if s["bias"] is None else out + s["bias"]).to(TYPES[c["to"]])
    if kind == "step":
        code = lambda v: _read8(*_float8(v), v.shape[1])  # noqa: E731
        x, w, dy, t = s["x"], s["w"], s["dy"], s["x"].dtype
        return {"y": (code(x) @ code(w).t()).to(t), "dx": (code(dy) @ code(w.t()).t()).to(t), "dw": code(dy.t()) @ code(x.t()).t()}
    t, x, h, mask = s["x"].dtype, s["x"].float(), s["h"].float(), _mask_of(s)
    if kind == "block":
        z = _affine(_normalise(x, c["pre"])[0], s["pre_gamma"], s["pre_beta"])
        z = z if c["act"] == "none" else z / (1 + torch.exp(-z))
        h = (_read8(*_float8(z), c["C"]) @ _load8(s["w"], c["C"]).t()).to(t).float()
    xo, z, stats = _join_plain(s, x, h, mask)
    out = {"xo": xo.to(t), "z": z.to(t)}
    if kind != "train":
        return out
    grads = _join_gradient(s, s["kept"].float(), h, s["kept_stats"], mask)
    for k in ("dx", "dh"):
        grads[k] = grads[k].to(t)
    return {**out, "stats": stats, **grads}


# ---- the framework's calls ------------------------------------------------------------------------
def _own(s):
    from paper_2006_09791_amd import binding as b
    c = s["case"]
    kind = c["kind"]
    if kind == "rows":
        b.gspc_quantize_rows_f8(s["x"], out=s["rows"], out_t=s["columns"])
        return {"rows": b.gspc_dequantize_rows_f8(s["rows"], c["cols"], out=s["out"]),
                "columns": b.gspc_dequantize_rows_f8(s["columns"], c["rows"], out=s["out_t"])}
    if kind == "dropout":
        return {"y": b.gspc_dropout(s["x"], c["drop"], s["seed"], s["offset"], out=s["y"]),
                "dx": b.gspc_dropout(s["dy"], c["drop"], s["seed"], s["offset"], out=s["dx"])}
    if kind == "linear":
        return b.gspc_matmul_f8(s["a"], s["w"], bias=s["bias"], out=s["out"])
    if kind == "step":
        for name in ("x", "w", "dy"):
            b.gspc_quantize_rows_f8(s[name], out=s[name + "8"], out_t=s[name + "8t"])
        return {"y": b.gspc_matmul_f8(s["x8"], s["w8"], out=s["y"]), "dx": b.gspc_matmul_f8(s["dy8"], s["w8t"], out=s["dx"]),
                "dw": b.gspc_matmul_f8(s["dy8t"], s["x8t"], out=s["dw"])}
    norms = {"none": b.NORM_NONE, "rms": b.NORM_RMS, "layer": b.NORM_LAYER}
    act = b.ACT_SILU if c["act"] == "silu" else b.ACT_NONE
    pre = {"pre": norms[c["pre"]], "pre_gamma": s["pre_gamma"], "pre_beta": s["pre_beta"], "act": act, "eps": EPS}
    both = {**pre, "post": norms[c["post"]], "post_gamma": s["post_gamma"], "post_beta": s["post_beta"], "gate": s["gate"],
            "scale": c["scale"], "drop": c["drop"], "seed": s["seed"], "offset": s["offset"]}
    if kind == "block":
        b.gspc_residual_norm(s["x"], None, out=s["z8"], **pre)
        b.gspc_matmul_f8(s["z8"], s["w"], out=s["h"])
    xo, z = b.gspc_residual_norm(s["x"], s["h"], xo=s["xo"], out=s["z"], stats=s.get("stats"), **both)
    if kind != "train":
        return {"xo": xo, "z": z}
    names = ("dx", "dh", "dgate", "dpost_gamma", "dpost_beta", "dpre_gamma", "dpre_beta")
    del both["eps"]
    b.gspc_residual_norm_backward(s["dz"], s["dxo"], s["kept"], s["h"], s["kept_stats"], **both, **{k: s[k] for k in names})
    return {"xo": xo, "z": z, "stats": s["stats"], **{k: s[k] for k in names if s[k] is not None}}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2}
    coded = lambda rows, cols: rows * (cols + -(-cols // 128))  # noqa: E731
    if kind == "rows":
        R, C, e = case["rows"], case["cols"], size[case["dtype"]]
        return {"bytes": 3 * R * C * e + 2 * (coded(R, C) + coded(C, R)), "flops": 6 * R * C}
    if kind == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 4 * n * size[case["dtype"]], "flops": 2 * n}
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": coded(M, K) + coded(N, K) + M * N * size[case["to"]] + (4 * N if case["bias"] else 0), "flops": 2 * M * K * N}
    if kind == "step":
        M, K, N = case["M"], case["K"], case["N"]
        both = sum(coded(a, b) + coded(b, a) for a, b in ((M, K), (N, K), (M, N)))     # written, and read by one product each
        return {"bytes": 2 * M * (K + N) + 4 * N * K + 2 * both + 2 * M * (N + K) + 4 * N * K, "flops": 6 * M * K * N}
    rows, C, e = case["N"] * case["P"], case["C"], size[case["dtype"]]
    n, vectors = rows * C, 4 * C * (4 + (case["N"] if case["gate"] == "image" else 1))
    if kind == "join":
        return {"bytes": 4 * n * e + vectors, "flops": 16 * n}
    if kind == "train":
        return {"bytes": 10 * n * e + 32 * rows + 3 * vectors, "flops": 48 * n}
    return {"bytes": n * e + 2 * coded(rows, C) + coded(C, C) + n * 2 + 4 * n * e + 2 * vectors, "flops": (24 + 2 * C) * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_pow2(k):
    """2^k in 64 bits, k a tensor of whole numbers."""
    return (k.long() + 1023 << 52).view(torch.float64)


def _exact8(x):
    """What x [rows, cols], in 64 bits, is read back as from 8-bit float rows."""
    rows, cols = x.shape
    blocks = torch.cat((x, x.new_zeros(rows, -cols % 128)), 1).reshape(rows, -1, 128)
    top = blocks.abs().max(-1, keepdim=True).values
    k = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448))
    k = torch.where(top > 448 * _exact_pow2(k), k + 1, torch.where(top <= 448 * _exact_pow2(k - 1), k - 1, k)).clamp(min=-127)
    v = blocks / _exact_pow2(k)
    size = v.abs()
    grid = torch.full_like(size, 2.0 ** -9)
    for e in range(-5, 9):                      # the distance of neighbours from 2^e on
        grid[size >= 2.0 ** e] = 2.0 ** (e - 3)
    return ((v / grid).round() * grid * _exact_pow2(k)).reshape(rows, -1)[:, :cols]


def _exact_mask(rows, cols, drop, seed, offset):
    """The same numbers, with products of 32 by 32 bits from products of 16 by 32."""
    low = (1 << 32) - 1

    def product(a, x):
        upper, lower = (a >> 16) * x, (a & 0xffff) * x
        return (upper + (lower >> 16)) >> 16, (((upper & 0xffff) << 16) + lower) & low

    block, row = torch.arange((cols + 7) // 8, device=DEVICE), torch.arange(rows, device=DEVICE)
    a, b = block.expand(rows, -1), row.unsqueeze(1).expand(-1, len(block))
    c, d = torch.full_like(a, offset % (1 << 32)), torch.full_like(a, offset >> 32)
    for i in range(10):
        key = ((seed & low) + i * 0x9E3779B9) & low, ((seed >> 32) + i * 0xBB67AE85) & low
        high_a, low_a = product(0xD2511F53, a)
        high_c, low_c = product(0xCD9E8D57, c)
        a, b, c, d = high_c ^ b ^ key[0], low_c, high_a ^ d ^ key[1], low_a
    numbers = torch.empty(rows, len(block), 8, dtype=torch.int64, device=DEVICE)
    for i, word in enumerate((a, b, c, d)):
        numbers[..., 2 * i], numbers[..., 2 * i + 1] = word % 65536, word // 65536
    limit = int(drop * 65536 + 0.5)
    return (numbers.reshape(rows, -1)[:, :cols] >= limit).double() * (65536 / (65536 - limit))


def _exact_norm(x, kind):
    """(x hat, mean, 1 / deviation)"""
    zero = x.new_zeros(x.shape[0], 1)
    if kind == "none":
        return x, zero, zero + 1
    mean = x.sum(1, keepdim=True) / x.shape[1] if kind == "layer" else zero
    rstd = ((x - mean).pow(2).sum(1, keepdim=True) / x.shape[1] + EPS).rsqrt()
    return (x - mean) * rstd, mean, rstd


def _exact_back(grad, xh, rstd, kind):
    if kind == "none":
        return grad
    n = xh.shape[1]
    centre = grad.sum(1, keepdim=True) / n if kind == "layer" else 0.0
    return rstd * (grad - centre - xh * ((grad * xh).sum(1, keepdim=True) / n))


def exact(case, seed):
    s = prepare(case, seed)
    kind, c = case["kind"], case
    up = lambda k: None if s[k] is None else s[k].double()  # noqa: E731
    if kind == "rows":
        return {"rows": _exact8(up("x")), "columns": _exact8(up("x").T.contiguous())}
    if kind == "dropout":
        m = _exact_mask(c["rows"], c["cols"], c["drop"], s["seed"], s["offset"])
        return {"y": up("x") * m, "dx": up("dy") * m}
    stored = lambda pair, cols: (pair[0].double() * _exact_pow2(pair[1][:, :pair[0].shape[1] // 128].long() - 127)  # noqa: E731
                                 .repeat_interleave(128, 1))[:, :cols]
    if kind == "linear":
        y = torch.matmul(stored(s["a"], c["K"]), stored(s["w"], c["K"]).T.contiguous())
        return y if s["bias"] is None else y + up("bias")
    if kind == "step":
        x, w, dy = up("x"), up("w"), up("dy")
        turned = lambda v: _exact8(v.T.contiguous())  # noqa: E731
        return {"y": torch.matmul(_exact8(x), _exact8(w).T.contiguous()), "dx": torch.matmul(_exact8(dy), turned(w).T.contiguous()),
                "dw": torch.matmul(turned(dy), turned(x).T.contiguous())}
    t, rows, C = TYPES[c["dtype"]], c["N"] * c["P"], c["C"]
    one, zero = torch.ones(C, device=DEVICE, dtype=torch.float64), torch.zeros(C, device=DEVICE, dtype=torch.float64)
    g1, b1, g2, b2 = (d if s[k] is None else up(k) for k, d in (("post_gamma", one), ("post_beta", zero), ("pre_gamma", one), ("pre_beta", zero)))
    gate = torch.ones(1, C, device=DEVICE, dtype=torch.float64) if s["gate"] is None else up("gate")
    gate = gate.unsqueeze(1).expand(-1, rows // gate.shape[0], -1).reshape(rows, C)
    x, h = up("x"), up("h")
    if kind == "block":
        z = _exact_norm(x, c["pre"])[0] * g2 + b2
        z = z * torch.sigmoid(z) if c["act"] == "silu" else z
        h = torch.matmul(_exact8(z), stored(s["w"], C).T.contiguous()).to(t).double()
    m = _exact_mask(rows, C, c["drop"], s["seed"], s["offset"]) if c["drop"] else 1.0
    hh, m1, r1 = _exact_norm(h, c["post"])
    u = (hh * g1 + b1) * m
    xo = c["scale"] * x + gate * u
    xh, m2, r2 = _exact_norm(xo, c["pre"])
    v = xh * g2 + b2
    out = {"xo": xo, "z": v * torch.sigmoid(v) if c["act"] == "silu" else v}
    if kind != "train":
        return out
    (k1, kr1, k2, kr2), stats = up("kept_stats").split(1, 1), torch.cat((m1, r1, m2, r2), 1)
    xh, hh, r1, r2 = (up("kept") - k2) * kr2, (h - k1) * kr1, kr1, kr2
    u = (hh * g1 + b1) * m
    v = xh * g2 + b2
    sig = torch.sigmoid(v)
    dv = up("dz") * (sig + v * sig * (1 - sig) if c["act"] == "silu" else 1.0)
    total = up("dxo") + _exact_back(dv * g2, xh, r2, c["pre"])
    du = total * gate * m
    grads = {"dx": c["scale"] * total, "dh": _exact_back(du * g1, hh, r1, c["post"]), "dpre_gamma": (dv * xh).sum(0)}
    if s["pre_beta"] is not None:
        grads["dpre_beta"] = dv.sum(0)
    if s["gate"] is not None:
        grads["dgate"] = (total * u).reshape(s["gate"].shape[0], -1, C).sum(1)
    if s["post_gamma"] is not None:
        grads["dpost_gamma"] = (du * hh).sum(0)
    if s["post_beta"] is not None:
        grads["dpost_beta"] = du.sum(0)
    return {**out, "stats": stats, **grads}
