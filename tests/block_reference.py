"""Definitions of a residual block's operators in 64 bits (numpy): 8-bit float rows, dropout's generator, the norms with gate and residual and their
gradient, with the magnitudes that errors are measured against."""
import contextlib

import numpy as np

U = 2.0 ** -24          # half a last place of fp32, relative
B = 2.0 ** -8           # ... of bf16


# ---- 8-bit float rows ----------------------------------------------------------------------------
def f8_reference(x):
    """x [rows, cols] (values that fp32 holds) -> (values [rows, pitch], NaN where x is not finite; bytes [rows, scale pitch])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    pitch = (cols + 127) // 128 * 128
    v = np.zeros((rows, pitch))
    v[:, :cols] = x
    v = v.reshape(rows, -1, 128)
    finite = np.isfinite(v)
    top = np.where(finite, np.abs(v), 0).max(2)
    m, e = np.frexp(top)                                        # top = m 2^e, m from 1/2
    k = np.where(top > 0, np.where(m > 0.875, e - 8, e - 9), -127)      # 448 = 7/8 2^9
    k = np.maximum(k, -127)
    with np.errstate(invalid="ignore"):
        w = np.ldexp(np.where(finite, v, 0), -k[:, :, None])
    step = np.ldexp(1.0, np.maximum(np.frexp(w)[1] - 1, -6) - 3)
    w = np.where(finite, np.rint(w / step) * step, np.nan)
    code = np.zeros((rows, (cols + 511) // 512 * 4), np.uint8)
    code[:, :k.shape[1]] = k + 127
    return w.reshape(rows, pitch), code


def f8_read(q, code):
    """What rows stand for, [rows, pitch]."""
    rows, pitch = q.shape
    k = code[:, :pitch // 128].astype(np.int64) - 127
    return (q.reshape(rows, -1, 128) * np.ldexp(1.0, k)[:, :, None]).reshape(rows, pitch)


# ---- dropout ---------------------------------------------------------------------------------------
def philox(c, key):
    """c: four arrays of 32-bit words, key: 64 bits -> four arrays (Philox 4x32-10)."""
    c = [np.asarray(w, np.uint64) for w in c]
    low = np.uint64(0xffffffff)
    k = [key & 0xffffffff, key >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def dropout_factors(rows, cols, drop, seed, offset):
    """What each value is multiplied by, in 64 bits; rows: their number, or the numbers of some."""
    limit = int(np.rint(drop * 65536))
    row, vec = np.meshgrid(np.arange(rows) if np.isscalar(rows) else np.asarray(rows), np.arange((cols + 7) // 8), indexing="ij")
    offset &= (1 << 64) - 1
    words = philox((vec, row, np.full_like(vec, offset & 0xffffffff), np.full_like(vec, offset >> 32)), seed)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xffff), w >> np.uint64(16))], 2).reshape(len(row), -1)[:, :cols]
    return np.where(halves >= limit, 65536.0 / max(1, 65536 - limit), 0.0)


# ---- norms with gate and residual --------------------------------------------------------------------
def act64(z, act):
    return z if act == 0 else np.maximum(z, 0) if act == 1 else z / (1 + np.exp(-z))


def slope64(z, act):
    s = 1 / (1 + np.exp(-z))
    return np.ones_like(z) if act == 0 else (z > 0).astype(float) if act == 1 else s * (1 + z * (1 - s))


def normalise(x, kind, eps):
    """(x hat, mean, 1 / deviation)"""
    mean = x.mean(1, keepdims=True) if kind == 2 else np.zeros((len(x), 1))
    if kind == 0:
        return x, mean, np.ones_like(mean)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd, mean, rstd


def each_row(gate, rows):
    return np.repeat(gate, rows // len(gate), 0)


def forward64(p, x, h):
    """p: dict of post, pre, act, scale, eps, the parameters (None for what is not there), gate [gates, C] or None, mask [rows, C] or None.
    -> dict of xo, z, stats, and the errors that are allowed before a result is rounded to its type.

    The errors: x - mean is rounded and so is the mean, 2 u (|xh| + |mean| rstd) of xh; the mean's and the variance's own sums, of differences in tree
    order over at most 8192 values, stay below 64 u of the spread; 256 u (1 + |xh| + |mean| rstd) leaves a factor of about two.  What x' is off by
    enters the second norm by itself and through its row's mean and deviation: at most the row's largest, times 2 + |xh|."""
    rows, C = x.shape
    one, zero = np.ones(C), np.zeros(C)
    g1, b1, g2, b2 = (d if p[k] is None else p[k] for k, d in (("post_gamma", one), ("post_beta", zero), ("pre_gamma", one), ("pre_beta", zero)))
    e_xo = 4 * U * np.abs(p["scale"] * x)
    xo, m1, r1 = p["scale"] * x, np.zeros((rows, 1)), np.ones((rows, 1))
    if h is not None:
        hh, m1, r1 = normalise(h, p["post"], p["eps"])
        u = hh * g1 + b1
        e_u = 4 * U * (np.abs(u) + np.abs(b1)) + (256 * U * (1 + np.abs(hh) + np.abs(m1) * r1) * np.abs(g1) if p["post"] else 0)
        w = (1 if p["gate"] is None else each_row(p["gate"], rows)) * (1 if p["mask"] is None else p["mask"])
        xo = xo + w * u
        e_xo = e_xo + np.abs(w) * e_u + 8 * U * np.abs(w * u) + U * np.abs(xo)
    xh, m2, r2 = normalise(xo, p["pre"], p["eps"])
    v = xh * g2 + b2
    far = e_xo.max(1, keepdims=True)
    e_v = np.abs(g2) * (256 * U * (1 + np.abs(xh) + np.abs(m2) * r2) + r2 * far * (2 + np.abs(xh))) + 4 * U * (np.abs(v) + np.abs(b2))
    return {"xo": xo, "z": act64(v, p["act"]), "stats": np.concatenate((m1, r1, m2, r2), 1), "e_xo": e_xo, "e_z": 1.1 * e_v + 16 * U * np.abs(v) + 1e-30,
            "far": far}


def backward64(p, dz, dxo, xo, h, stats):
    """-> {name: (gradient, magnitudes of what it is the sum of)}; errors are taken as 256 u of the latter (chains of at most 1024 terms, joined in
    trees or in 64 bits, and a handful of roundings each)."""
    rows, C = xo.shape
    one, zero = np.ones(C), np.zeros(C)
    g1, b1, g2, b2 = (d if p[k] is None else p[k] for k, d in (("post_gamma", one), ("post_beta", zero), ("pre_gamma", one), ("pre_beta", zero)))
    m1, r1, m2, r2 = (stats[:, k:k + 1] for k in range(4))
    mean = lambda a: a.mean(1, keepdims=True)  # noqa: E731
    out = {}
    dX, size = (np.zeros_like(xo),) * 2 if dxo is None else (dxo, np.abs(dxo))
    if dz is not None:
        xh, XH = (xo - m2) * r2, (np.abs(xo) + np.abs(m2)) * r2
        v = xh * g2 + b2
        dv, DV = dz * slope64(v, p["act"]), np.abs(dz) * (1.1 + (XH * np.abs(g2) + np.abs(b2) if p["act"] else 0))
        t, T = dv * g2, DV * np.abs(g2)
        dX = dX + r2 * (t - (mean(t) if p["pre"] == 2 else 0) - xh * mean(t * xh))
        size = size + r2 * (T + (mean(T) if p["pre"] == 2 else 0) + XH * mean(T * XH))
        out["dpre_gamma"], out["dpre_beta"] = ((dv * xh).sum(0), (DV * XH).sum(0)), (dv.sum(0), DV.sum(0))
    out["dx"] = p["scale"] * dX, np.abs(p["scale"]) * size
    if h is not None:
        hh, HH = (h - m1) * r1, (np.abs(h) + np.abs(m1)) * r1
        gate = np.ones((1, C)) if p["gate"] is None else p["gate"]
        mask = 1.0 if p["mask"] is None else p["mask"]
        d, D = dX * mask, size * mask
        wide = each_row(gate, rows)
        q, Q = d * wide * g1, D * np.abs(wide * g1)
        out["dh"] = (q, Q) if p["post"] == 0 else (r1 * (q - (mean(q) if p["post"] == 2 else 0) - hh * mean(q * hh)),
                                                   r1 * (Q + (mean(Q) if p["post"] == 2 else 0) + HH * mean(Q * HH)))
        per = lambda a: a.reshape(len(gate), -1, C).sum(1)  # noqa: E731
        out["dgate"] = per(d * (hh * g1 + b1)), per(D * (HH * np.abs(g1) + np.abs(b1)))
        out["dpost_gamma"] = (d * wide * hh).sum(0), (D * np.abs(wide) * HH).sum(0)
        out["dpost_beta"] = (d * wide).sum(0), (D * np.abs(wide)).sum(0)
    return out


@contextlib.contextmanager
def on_side_stream(torch, b):
    """torch and the library on a stream that is not the default one, which is yielded."""
    from helpers import side_stream
    stream = side_stream()
    torch.cuda.synchronize()
    try:
        with torch.cuda.stream(stream):
            b.gspc_set_stream()
            yield stream
            stream.synchronize()
    finally:
        b.gspc_set_stream(torch.cuda.default_stream())
