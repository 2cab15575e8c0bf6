"""Channels-last operators on the GPU against their definitions in 64 bits (numpy): layout passes, 8-bit rows, group norm with an
activation and its gradient, products of 8-bit rows.

Tolerances, with u = 2^-24 (fp32) and 2^-8 for a value rounded to bf16 (half of its last place is 2^-9 to 2^-8 of it):
  group norm: x - mean is rounded and so is the mean, u (|x| + |mean|) rstd <= 2 u (|xh| + |mean| rstd) of xh; the mean's and the
  variance's own sums, of differences and in tree order, stay below 64 u of the group's spread (chains of at most 32 terms behind
  one another, joined in trees).  SiLU's slope is below 1.1 and its own rounding a few u.  Together 256 u (1 + |xh| + |mean| rstd)
  |gamma| leaves a factor of about two.
  gradient: sums of n terms over up to 128 chunks; their error is taken as 256 u of the sum of magnitudes.
"""
import numpy as np
import pytest

from helpers import side_stream
from test_gpu_parity import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B = 2.0 ** -8


def dev(torch, a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy()


def strided(torch, x, extra):
    """x as some channels of a wider tensor, the rest NaN."""
    wide = torch.full((*x.shape[:-1], x.shape[-1] + extra), float("nan"), dtype=x.dtype, device=x.device)
    view = wide[..., extra // 2:extra // 2 + x.shape[-1]]
    view.copy_(x)
    return wide, view


# ---- layout --------------------------------------------------------------------------------------
@pytest.mark.parametrize("N,C,P", [(1, 1, 1), (2, 3, 5), (3, 7, 64), (1, 8, 8), (2, 9, 65), (5, 84, 1073), (3, 64, 49), (2, 130, 63),
                                   (1, 512, 1), (300, 2, 3), (1, 1, 200), (4, 200, 7)])
@pytest.mark.parametrize("src", ["float32", "bfloat16"])
@pytest.mark.parametrize("dst", ["float32", "bfloat16"])
def test_layout(gpu, N, C, P, src, dst):
    torch, b = gpu
    x = torch.randn(N, C, P, device="cuda").to(getattr(torch, src))
    kind = {"float32": b.GSPC_F32, "bfloat16": b.GSPC_BF16}[dst]
    y = b.gspc_pack_channels_last(x, dtype=kind)
    assert y.shape == (N, P, C) and torch.equal(y, x.transpose(1, 2).to(getattr(torch, dst)))
    z = b.gspc_unpack_channels_last(y, dtype=b.GSPC_F32)
    assert z.shape == (N, C, P) and torch.equal(z, y.transpose(1, 2).float())


# ---- 8-bit rows ----------------------------------------------------------------------------------
def rows8_reference(x):
    """The definition's own operations in fp32, each rounded once: integers have to be equal."""
    x = x.astype(np.float32)
    top = np.abs(x).max(1, keepdims=True)
    with np.errstate(all="ignore"):
        up = np.where(top < np.float32(2.0 ** -64), np.float32(2.0 ** 64), np.float32(1))
        inv = np.where(top > 0, np.float32(127) / (top * up), np.float32(0))
        q = np.rint((x * up) * inv)
        scale = (top / np.float32(127))[:, 0]
    bad = ~np.isfinite(x).all(1)
    q[bad], scale[bad] = 0, np.nan
    return q.astype(np.int8), scale


@pytest.mark.parametrize("cols", [1, 2, 7, 8, 9, 15, 16, 17, 60, 64, 333, 511, 512, 513, 1000, 1024, 1500, 2049, 4096, 4104, 5003])
@pytest.mark.parametrize("rows", [1, 3, 130])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows8(gpu, cols, rows, dtype):
    torch, b = gpu
    rng = np.random.default_rng(cols * 1000 + rows)
    x = rng.standard_normal((rows, cols)).astype(np.float32) * np.float32(2.0) ** rng.integers(-12, 12, (rows, 1))
    if rows > 100:
        x[3] = 0
        x[5] *= np.float32(1e-30)
        x[6] = np.float32(2.0 ** -149) * rng.integers(-3, 4, cols)     # the smallest numbers there are
        x[7] *= np.float32(2.0 ** 100)
        x[8, -1] = np.inf
        x[9, 0] = np.nan
        x[10, cols // 2] = -np.inf
        x[11] = 1.5                                                    # all at the end of the range
        x[12] = -127 * np.float32(2.0 ** -140)                         # a scale that is no normal number
        x[13] = np.float32(3.4e38)
        x[14, :] = (np.arange(cols) % 255 - 127) / 2.0 * 2 ** 3        # halves: ties
        x[14, 0] = 127 * 2.0 ** 3
    t = dev(torch, x, getattr(torch, dtype))
    wide, view = strided(torch, t, 6)
    want_q, want_s = rows8_reference(t.float().cpu().numpy())
    for src in (t, view):
        pitch = b.gspc_rows8_pitch(cols)
        q = torch.full((rows + 2, pitch), 77, dtype=torch.int8, device="cuda")
        s = torch.full((rows + 2,), 7.0, device="cuda")
        b.gspc_quantize_rows(src, out=(q[1:-1], s[1:-1]))
        got = q.cpu().numpy()
        assert (got[0] == 77).all() and (got[-1] == 77).all() and s[0] == s[-1] == 7
        assert np.array_equal(got[1:-1, :cols], want_q) and (got[1:-1, cols:] == 0).all()
        assert np.array_equal(s[1:-1].cpu().numpy(), want_s, equal_nan=True)
        back = torch.full((rows, cols + 6), 5.0, dtype=t.dtype, device="cuda")
        b.gspc_dequantize_rows((q[1:-1], s[1:-1]), cols, out=back[:, 3:-3])
        want = (torch.from_numpy(want_q).float() * torch.from_numpy(want_s)[:, None]).to(t.dtype)
        assert torch.equal(torch.nan_to_num(back[:, 3:-3].cpu(), nan=-1), torch.nan_to_num(want, nan=-1))
        assert (back[:, :3] == 5).all() and (back[:, -3:] == 5).all()


def test_rows8_of_nothing(gpu):
    torch, b = gpu
    q, s = b.gspc_quantize_rows(torch.zeros(0, 40, device="cuda"))
    assert q.shape == (0, 48) and s.shape == (0,)
    assert b.gspc_dequantize_rows((q, s), 40).shape == (0, 40)


# ---- group norm ----------------------------------------------------------------------------------
def act64(z, act):
    return z if act == 0 else np.maximum(z, 0) if act == 1 else z / (1 + np.exp(-z))


def slope64(z, act):
    s = 1 / (1 + np.exp(-z))
    return np.ones_like(z) if act == 0 else (z > 0).astype(float) if act == 1 else s * (1 + z * (1 - s))


def norm64(x, gamma, beta, groups, eps):
    """(xh, z, mean per value, rstd per value, stats) in 64 bits."""
    N, P, C = x.shape
    v = x.reshape(N, P, groups, C // groups)
    mean = v.mean((1, 3), keepdims=True)
    rstd = 1 / np.sqrt(((v - mean) ** 2).mean((1, 3), keepdims=True) + eps)
    xh = (v - mean) * rstd
    spread = lambda a: np.broadcast_to(a, v.shape).reshape(x.shape)  # noqa: E731
    xh = xh.reshape(x.shape)
    return xh, xh * gamma + beta, spread(mean), spread(rstd), np.stack((mean[:, 0, :, 0], rstd[:, 0, :, 0]), 2)


def grad64(dy, x, stats, gamma, beta, groups, act):
    """(dx, dgamma, dbeta) and the sums of magnitudes that their errors are measured against."""
    N, P, C = x.shape
    D = C // groups
    mean, rstd = (np.repeat(stats[..., k], D, 1)[:, None] for k in (0, 1))
    xh = (x - mean) * rstd
    dz = dy * slope64(xh * gamma + beta, act)
    t = dz * gamma
    per = lambda a: np.repeat(a.reshape(N, P, groups, D).mean((1, 3)), D, 1)[:, None]  # noqa: E731
    dx = rstd * (t - per(t) - xh * per(t * xh))
    size = rstd * (np.abs(t) + per(np.abs(t)) + np.abs(xh) * per(np.abs(t * xh)))
    return dx, (dz * xh).sum((0, 1)), dz.sum((0, 1)), size, np.abs(dz * xh).sum((0, 1)), np.abs(dz).sum((0, 1)), xh, mean * rstd


SHAPES = [  # N, P, C, groups: one value a group; fewer than eight channels; sizes off every vector; several slabs of channels, with a
    # group across their border and a last slab of two channels; long thin and wide short ones
    (1, 1, 1, 1), (2, 1, 8, 8), (3, 1, 64, 4), (2, 5, 3, 1), (2, 17, 6, 3), (1, 9, 7, 7), (5, 63, 60, 3), (2, 49, 512, 32), (3, 50, 96, 96),
    (1, 7, 2050, 2), (2, 6, 4100, 4), (1, 3, 2500, 1), (1, 20, 2048, 2048), (1, 12544, 16, 2), (4, 200, 130, 13), (70, 4, 32, 8), (2, 300, 1280, 32),
    (1, 1000, 33, 1), (300, 2, 24, 3), (1, 70000, 8, 1),
]


def norm_inputs(N, P, C, seed, offset=0.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, P, C)) * np.exp(0.5 * rng.standard_normal(C)) + 0.5 * rng.standard_normal(C) + offset
    return x.astype(np.float32), (1 + 0.2 * rng.standard_normal(C)).astype(np.float32), (0.2 * rng.standard_normal(C)).astype(np.float32)


def norm_tol(xh, z, mean, rstd, gamma, y, bf16):
    return 256 * U * (1 + np.abs(xh) + np.abs(mean) * rstd) * (np.abs(gamma) + np.abs(z)) + (B * np.abs(y) if bf16 else 0) + 1e-30


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("src,dst", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("bfloat16", "float32")])
def test_norm(gpu, shape, src, dst):
    torch, b = gpu
    N, P, C, groups = shape
    x, gamma, beta = norm_inputs(N, P, C, N + P + C)
    xd = dev(torch, x, getattr(torch, src))
    x = host(xd)
    act = (N + P + C) % 3
    xh, z, mean, rstd, stats = norm64(x, gamma.astype(float), beta.astype(float), groups, 1e-5)
    y = act64(z, act)
    tol = norm_tol(xh, z, mean, rstd, gamma, y, dst == "bfloat16")
    st = torch.full((N, groups, 2), 9.0, device="cuda")
    _, xs = strided(torch, xd, 10)
    wide, ys = strided(torch, torch.zeros(N, P, C, dtype=getattr(torch, dst), device="cuda"), 6)
    plain = torch.empty(N, P, C, dtype=getattr(torch, dst), device="cuda")
    b.gspc_group_norm(xd, dev(torch, gamma), dev(torch, beta), groups, 1e-5, act, out=plain, stats=st)
    b.gspc_group_norm(xs, dev(torch, gamma), dev(torch, beta), groups, 1e-5, act, out=ys)
    assert (np.abs(host(plain) - y) <= tol).all(), np.max(np.abs(host(plain) - y) / tol)
    assert torch.equal(plain, ys) and bool(wide[..., :3].isnan().all()) and bool(wide[..., -3:].isnan().all())
    st = host(st)
    assert (np.abs(st[..., 0] - stats[..., 0]) * stats[..., 1] <= 256 * U * (1 + np.abs(stats[..., 0]) * stats[..., 1])).all()
    assert (np.abs(st[..., 1] / stats[..., 1] - 1) <= 256 * U * (1 + np.abs(stats[..., 0]) * stats[..., 1])).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("src", ["float32", "bfloat16"])
def test_norm_to_rows8_and_saved(gpu, shape, src):
    """y as 8-bit rows: within half a step (and the row's own error) of y.  saved: exactly what gspc_quantize_rows writes."""
    torch, b = gpu
    N, P, C, groups = shape
    x, gamma, beta = norm_inputs(N, P, C, 7 * N + P + C)
    xd = dev(torch, x, getattr(torch, src))
    act = (N + P + C + 1) % 3
    xh, z, mean, rstd, _ = norm64(host(xd), gamma.astype(float), beta.astype(float), groups, 1e-5)
    y = act64(z, act).reshape(N * P, C)
    tol = norm_tol(xh, z, mean, rstd, gamma, 0, False).reshape(N * P, C)
    pitch = b.gspc_rows8_pitch(C)
    for save in (False, True):
        q, s, sq, ss = (torch.full((N * P + 1, pitch), 55, dtype=torch.int8, device="cuda"), torch.zeros(N * P, device="cuda"),
                        torch.full((N * P, pitch), 55, dtype=torch.int8, device="cuda"), torch.zeros(N * P, device="cuda"))
        b.gspc_group_norm(xd, dev(torch, gamma), dev(torch, beta), groups, 1e-5, act, out=(q[:-1], s), saved=(sq, ss) if save else None)
        assert (q[-1] == 55).all() and (q[:-1, C:] == 0).all()
        step = np.abs(y).max(1, keepdims=True) / 127
        err = np.abs(host(q[:-1, :C]) * host(s)[:, None] - y)
        row_tol = tol.max(1, keepdims=True)
        assert (err <= 0.501 * step + 2 * tol + row_tol).all()
        assert (np.abs(host(s)[:, None] - step) <= row_tol + 4 * U * step).all()
        if save:
            want = b.gspc_quantize_rows(xd)
            assert torch.equal(sq, want[0]) and torch.equal(ss, want[1])
            sq.fill_(55)
            ss.zero_()
            out = b.gspc_group_norm(xd, dev(torch, gamma), dev(torch, beta), groups, 1e-5, act, saved=(sq, ss))
            assert torch.equal(sq, want[0]) and torch.equal(ss, want[1])
            assert torch.equal(out, b.gspc_group_norm(xd, dev(torch, gamma), dev(torch, beta), groups, 1e-5, act))


@pytest.mark.parametrize("shape", [(2, 400, 32, 4), (1, 30, 2050, 2), (3, 49, 64, 32)], ids=str)
def test_norm_offsets_and_outliers(gpu, shape):
    """An offset far above the spread, and a first value far from all others: the variance is not a difference of large sums."""
    torch, b = gpu
    N, P, C, groups = shape
    for offset, outlier in ((1000.0, 0), (0.0, 3e4), (-300.0, -1e4)):
        x, gamma, beta = norm_inputs(N, P, C, 3, offset)
        if outlier:
            x[:, 0, 0] = outlier
        xh, z, mean, rstd, _ = norm64(x.astype(float), gamma.astype(float), beta.astype(float), groups, 1e-5)
        y = host(b.gspc_group_norm(dev(torch, x), dev(torch, gamma), dev(torch, beta), groups, 1e-5, b.ACT_NONE))
        tol = norm_tol(xh, z, mean, rstd, gamma, z, False)
        assert (np.abs(y - z) <= tol).all(), np.max(np.abs(y - z) / tol)


def test_norm_without_spread_or_parameters(gpu):
    """A constant group: the variance is zero and y is beta.  No gamma, no beta: 1 and 0."""
    torch, b = gpu
    x = torch.full((2, 50, 24), 3.25, device="cuda")
    beta = torch.randn(24, device="cuda")
    assert torch.equal(b.gspc_group_norm(x, None, beta, 3), beta.expand(2, 50, 24))
    x = torch.randn(2, 50, 24, device="cuda")
    one, zero = torch.ones(24, device="cuda"), torch.zeros(24, device="cuda")
    assert torch.equal(b.gspc_group_norm(x, None, None, 3), b.gspc_group_norm(x, one, zero, 3))
    dy, st = torch.randn(2, 50, 24, device="cuda"), torch.empty(2, 3, 2, device="cuda")
    b.gspc_group_norm(x, None, None, 3, stats=st)
    for p, q in zip(b.gspc_group_norm_backward(dy, x, st, None, None, 3, b.ACT_SILU), b.gspc_group_norm_backward(dy, x, st, one, zero, 3, b.ACT_SILU)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("pixels", [40, 9001])      # an image that a block holds, and one in two passes
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_keeps_what_is_not_finite_in_its_group(gpu, bad, pixels):
    torch, b = gpu
    x, gamma, beta = norm_inputs(3, pixels, 48, 4)
    x = dev(torch, x)
    clean = b.gspc_group_norm(x, dev(torch, gamma), dev(torch, beta), 6, act=b.ACT_RELU)
    x[1, 13, 17] = bad
    y = b.gspc_group_norm(x, dev(torch, gamma), dev(torch, beta), 6, act=b.ACT_RELU)
    assert bool(y[1, :, 16:24].isnan().all())
    y[1, :, 16:24] = clean[1, :, 16:24]
    assert torch.equal(y, clean)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kept,grad", [("float32", "float32"), ("bfloat16", "bfloat16"), ("rows8", "float32"), ("rows8", "bfloat16"),
                                       ("bfloat16", "float32"), ("float32", "bfloat16")])
def test_norm_backward(gpu, shape, kept, grad):
    torch, b = gpu
    N, P, C, groups = shape
    rng = np.random.default_rng(N + 3 * P + C)
    x, gamma, beta = norm_inputs(N, P, C, N + 2 * P + C)
    xd = dev(torch, x, torch.bfloat16 if kept == "bfloat16" else None)
    dyd = dev(torch, rng.standard_normal((N, P, C)).astype(np.float32), getattr(torch, grad))
    gd, bd, st = dev(torch, gamma), dev(torch, beta), torch.empty(N, groups, 2, device="cuda")
    act = (0, 2, 1)[(N + P + C) % 3]
    b.gspc_group_norm(xd, gd, bd, groups, 1e-5, act, stats=st)
    if kept == "rows8":
        q, s = b.gspc_quantize_rows(xd)
        x64, keep = (host(q)[:, :C] * host(s)[:, None]).reshape(N, P, C), (q, s)
    else:
        x64, keep = host(xd), xd
    dx, dgamma, dbeta, size, size_g, size_b, xh, shift = grad64(host(dyd), x64, host(st), gamma.astype(float), beta.astype(float), groups, act)
    got = b.gspc_group_norm_backward(dyd, keep, st, gd, bd, groups, act)
    tol = 256 * U * size * (1 + np.abs(xh) + np.abs(shift)) + (B * np.abs(dx) if grad == "bfloat16" else 0) + 1e-30
    near = np.zeros(dx.shape, bool)
    rel = 1 + np.abs(shift).max()
    if act == 1:        # values within rounding of the jump have no slope to speak of
        z = xh * gamma + beta
        near = np.abs(z) <= 16 * U * (1 + np.abs(xh) + np.abs(shift)) * (np.abs(gamma) + np.abs(beta))
        assert near.mean() < 1e-3
        loose = np.broadcast_to(np.where(near, np.abs(host(dyd)) * np.abs(gamma) * (1 + np.abs(xh)), 0).sum((0, 1)), C)
        tol = np.where(near, np.inf, tol + loose.max() * size.max() * near.any())
        size_g, size_b = size_g + loose / (256 * U * rel), size_b + loose / (256 * U * rel)
    assert (np.abs(host(got[0]) - dx) <= tol).all(), np.nanmax(np.abs(host(got[0]) - dx) / tol)
    assert (np.abs(host(got[1]) - dgamma) <= 256 * U * rel * size_g + 1e-30).all()
    assert (np.abs(host(got[2]) - dbeta) <= 256 * U * rel * size_b + 1e-30).all()
    # strides of all three, and gradients of parameters that nobody asked for
    _, gs = strided(torch, dyd, 4)
    wide, ds = strided(torch, torch.zeros_like(dyd), 12)
    if kept != "rows8":
        keep = strided(torch, xd, 2)[1]
    b.gspc_group_norm_backward(gs, keep, st, gd, bd, groups, act, dx=ds)
    assert torch.equal(ds, got[0]) and bool(wide[..., :6].isnan().all()) and bool(wide[..., -6:].isnan().all())


@pytest.mark.parametrize("act", [0, 2])
def test_norm_gradient_against_differences(gpu, act):
    """Along random directions: (L(+h) - L(-h)) / 2h with L = sum dy y, the forward's y in fp32.  The difference's own error: h^2 / 6
    times a third derivative of the order of L's terms, and rounding u sum |dy y| / h: with h = 2^-7 below 1e-3 of the norms."""
    torch, b = gpu
    N, P, C, groups = 2, 37, 40, 5
    x, gamma, beta = norm_inputs(N, P, C, 11)
    rng = np.random.default_rng(12)
    dy = rng.standard_normal((N, P, C)).astype(np.float32)
    gd, bd, dyd = dev(torch, gamma), dev(torch, beta), dev(torch, dy)
    st = torch.empty(N, groups, 2, device="cuda")
    b.gspc_group_norm(dev(torch, x), gd, bd, groups, 1e-5, act, stats=st)
    grads = [host(t) for t in b.gspc_group_norm_backward(dyd, dev(torch, x), st, gd, bd, groups, act)]
    h = 2.0 ** -7
    for at, base in enumerate((x, gamma, beta)):
        v = rng.standard_normal(base.shape).astype(np.float32)
        side = []
        for sign in (h, -h):
            args = [x, gamma, beta]
            args[at] = (base.astype(float) + sign * v).astype(np.float32)
            y = b.gspc_group_norm(dev(torch, args[0]), dev(torch, args[1]), dev(torch, args[2]), groups, 1e-5, act)
            side.append(float((host(y) * dy).sum()))
        along = (side[0] - side[1]) / (2 * h)
        want = float((grads[at] * v).sum())
        assert abs(along - want) <= 2e-3 * np.linalg.norm(grads[at]) * np.linalg.norm(v) / np.sqrt(v.size) * 4, (at, along, want)


def test_norm_of_nothing(gpu):
    torch, b = gpu
    for shape in ((0, 5, 16), (3, 0, 16)):
        x = torch.zeros(shape, device="cuda")
        assert b.gspc_group_norm(x, None, None, 4).shape == shape
        dg, db = torch.full((16,), 5.0, device="cuda"), torch.full((16,), 5.0, device="cuda")
        b.gspc_group_norm_backward(x, x, torch.zeros(shape[0], 4, 2, device="cuda"), None, None, 4, dgamma=dg, dbeta=db)
        assert not dg.any() and not db.any()


# ---- products ------------------------------------------------------------------------------------
def random_rows8(torch, rng, rows, cols, one=False):
    q = np.zeros((rows, (cols + 15) // 16 * 16), np.int8)
    q[:, :cols] = rng.integers(-127, 128, (rows, cols))
    s = np.ones(rows, np.float32) if one else np.exp(rng.standard_normal(rows)).astype(np.float32) / 127
    return q, s, (dev(torch, q), dev(torch, s))


SIZES = [(1, 1, 1), (1, 17, 16), (2, 15, 100), (15, 16, 17), (16, 33, 4096), (1, 1001, 1280), (7, 64, 333), (17, 100, 63), (33, 31, 64), (64, 64, 65),
         (100, 257, 129), (197, 1001, 1280), (130, 128, 127), (500, 500, 80), (2048, 2050, 272), (2100, 2049, 128), (4097, 4099, 144),
         (8200, 260, 4112), (300, 9000, 400), (5000, 16, 64), (20000, 40, 48), (16, 20000, 128)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_product_is_exact(gpu, M, N, K):
    """Scales of one: the integer sums, which fp32 holds while they stay below 2^24 (and rounds once beyond)."""
    torch, b = gpu
    rng = np.random.default_rng(M + N + K)
    qa, _, a = random_rows8(torch, rng, M, K, True)
    qw, _, w = random_rows8(torch, rng, N, K, True)
    want = qa.astype(np.float64) @ qw.astype(np.float64).T
    out = torch.full((M + 2, N + 5), 7.0, device="cuda")
    b.gspc_matmul_i8(a, w, out=out[1:-1, 2:-3])
    got = out.cpu().numpy()
    assert np.array_equal(got[1:-1, 2:-3], want.astype(np.float32)), b.gspc_last_kernel()
    edge = np.ones(got.shape, bool)
    edge[1:-1, 2:-3] = False
    assert (got[edge] == 7).all()
    got = b.gspc_matmul_i8(a, w, dtype=b.GSPC_BF16)
    assert torch.equal(got.cpu(), torch.from_numpy(want.astype(np.float32)).bfloat16())


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_product_scales_and_bias(gpu, M, N, K, dtype):
    """The sum rounded to fp32, two products and the bias: four roundings."""
    torch, b = gpu
    rng = np.random.default_rng(M + 2 * N + K)
    qa, sa, a = random_rows8(torch, rng, M, K)
    qw, sw, w = random_rows8(torch, rng, N, K)
    bias = rng.standard_normal(N).astype(np.float32)
    for bb in (None, bias):
        want = (qa.astype(np.float64) @ qw.astype(np.float64).T) * sa[:, None].astype(float) * sw.astype(float) + (0 if bb is None else bb.astype(float))
        got = b.gspc_matmul_i8(a, w, bias=None if bb is None else dev(torch, bb), out=torch.empty(M, N, dtype=getattr(torch, dtype), device="cuda"))
        tol = 4 * U * (np.abs(want) + (0 if bb is None else 2 * np.abs(bb))) + (B * np.abs(want) if dtype == "bfloat16" else 0) + 1e-30
        assert (np.abs(host(got) - want) <= tol).all(), b.gspc_last_kernel()


@pytest.mark.parametrize("M,N", [(1, 20), (40, 40), (2100, 2060)])
def test_product_longest_sum(gpu, M, N):
    """127 * 127 * 133144 is the largest sum that 32 bits hold; a row of NaN scale is NaN, and no other row is."""
    torch, b = gpu
    K = 133144 if M < 100 else 2000
    a = (torch.full((M, b.gspc_rows8_pitch(K)), 127, dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda"))
    w = (torch.full((N, b.gspc_rows8_pitch(K)), -127, dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda"))
    a[0][:, K:] = 0
    w[0][:, K:] = 0
    a[1][0] = float("nan")
    lib = b.load()
    out = torch.empty(M, N, device="cuda")
    assert lib.gspc_matmul_i8(a[0].data_ptr(), a[1].data_ptr(), w[0].data_ptr(), w[1].data_ptr(), None, M, N, K, out.data_ptr(), 0, N) == 0
    assert bool(out[0].isnan().all()) and bool((out[1:] == float(np.float32(-127.0 * 127 * K))).all())


def test_product_of_no_tokens(gpu):
    torch, b = gpu
    w = (torch.zeros(5, 16, dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda"))
    assert b.gspc_matmul_i8((torch.zeros(0, 16, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda")), w).shape == (0, 5)


# ---- together, on other streams, in graphs, and past 32 bits ---------------------------------------
def block(torch, b, x, dy, gamma, beta, groups, w, keep):
    """A training pass and an answering one through every operator of the set."""
    tokens = b.gspc_pack_channels_last(x, out=keep["tokens"])
    y = b.gspc_group_norm(tokens, gamma, beta, groups, act=b.ACT_SILU, out=keep["y"], stats=keep["stats"], saved=keep["saved"], workspace=keep["ws"])
    dx, dg, db = b.gspc_group_norm_backward(dy, keep["saved"], keep["stats"], gamma, beta, groups, b.ACT_SILU, dx=keep["dx"], dgamma=keep["dg"],
                                            dbeta=keep["db"], workspace=keep["ws"])
    q = b.gspc_group_norm(tokens, gamma, beta, groups, act=b.ACT_SILU, out=keep["q"], workspace=keep["ws"])
    out = b.gspc_matmul_i8(q, w, out=keep["out"])
    return [y, dx, dg, db, out, b.gspc_unpack_channels_last(out.view(*y.shape[:2], -1), out=keep["planes"])]


def block_inputs(torch, b, seed, N=3, C=48, P=70, cols=33):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    return (r(N, C, P), r(N, P, C).bfloat16(), r(C), r(C), 6, b.gspc_quantize_rows(r(cols, C)))


def block_buffers(torch, b, N=3, C=48, P=70, cols=33):
    e = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    rows8 = lambda: (e(N * P, b.gspc_rows8_pitch(C), t=torch.int8), e(N * P))  # noqa: E731
    size = max(b.gspc_group_norm_workspace_bytes(N, P, C, 6, b.GSPC_BF16, True),
               b.gspc_group_norm_backward_workspace_bytes(N, P, C, 6, b.GSPC_BF16, b.GSPC_I8))
    return {"tokens": e(N, P, C, t=torch.bfloat16), "y": e(N, P, C, t=torch.bfloat16), "stats": e(N, 6, 2), "saved": rows8(), "q": rows8(),
            "dx": e(N, P, C, t=torch.bfloat16), "dg": e(C), "db": e(C), "out": e(N, P, cols, t=torch.bfloat16), "planes": e(N, cols, P),
            "ws": e(size, t=torch.uint8)}


def test_block_on_a_side_stream_and_in_a_graph(gpu):
    torch, b = gpu
    inputs = [block_inputs(torch, b, s) for s in (1, 2)]
    want = [[t.clone() for t in block(torch, b, *i, block_buffers(torch, b))] for i in inputs]
    stream = side_stream()
    try:
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            b.gspc_set_stream()
            none = dict.fromkeys(block_buffers(torch, b))
            keep = dict(none, saved=block_buffers(torch, b)["saved"], q=block_buffers(torch, b)["q"], stats=torch.empty(3, 6, 2, device="cuda"))
            for i, w in zip(inputs, want):          # outputs and workspaces that the binding allocates
                got = block(torch, b, *i, keep)
                stream.synchronize()
                assert all(torch.equal(p.reshape(-1), q.reshape(-1).to(p.dtype)) for p, q in zip(got, w))
            held, keep = [t.clone() if torch.is_tensor(t) else t for t in block_inputs(torch, b, 1)], block_buffers(torch, b)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                b.gspc_set_stream()
                got = block(torch, b, *held, keep)
            for k in (0, 1, 0, 1):                  # new inputs in the recorded buffers
                for t, new in zip(held, inputs[k]):
                    if torch.is_tensor(t):
                        t.copy_(new)
                held[5][0].copy_(inputs[k][5][0])
                held[5][1].copy_(inputs[k][5][1])
                graph.replay()
                stream.synchronize()
                assert all(torch.equal(p, q) for p, q in zip(got, want[k]))
    finally:
        b.gspc_set_stream(torch.cuda.default_stream())


def test_same_call_same_bits(gpu):
    torch, b = gpu
    i = block_inputs(torch, b, 5)
    first = [t.clone() for t in block(torch, b, *i, block_buffers(torch, b))]
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, block(torch, b, *i, block_buffers(torch, b))))


def test_rows_past_32_bits(gpu):
    """Rows 2^20 elements apart: the last ones start beyond 2^32 elements."""
    torch, b = gpu
    rows, ld, C = 4200, 1 << 20, 40
    wide = torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda")
    x = wide[:, 16:16 + C]
    small = torch.randn(rows, C, device="cuda").bfloat16()
    x.copy_(small)
    q, s = b.gspc_quantize_rows(x)
    want = b.gspc_quantize_rows(small)
    assert torch.equal(q, want[0]) and torch.equal(s, want[1])
    y = wide[:, 512:512 + C]
    b.gspc_dequantize_rows(want, C, out=y)
    assert torch.equal(y, b.gspc_dequantize_rows(want, C, dtype=b.GSPC_BF16))
    images, view, out = small.view(3, 1400, C), x.unflatten(0, (3, 1400)), y.unflatten(0, (3, 1400))
    b.gspc_group_norm(view, None, None, 5, act=b.ACT_SILU, out=out)
    assert torch.equal(out, b.gspc_group_norm(images, None, None, 5, act=b.ACT_SILU))
    st = torch.empty(3, 5, 2, device="cuda")
    b.gspc_group_norm(images, None, None, 5, stats=st)
    want = b.gspc_group_norm_backward(images, images, st, None, None, 5, b.ACT_SILU)
    got = b.gspc_group_norm_backward(view, view, st, None, None, 5, b.ACT_SILU, dx=out)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    a = (torch.randint(-127, 128, (rows, 48), dtype=torch.int8, device="cuda"), torch.rand(rows, device="cuda"))
    w = (torch.randint(-127, 128, (C, 48), dtype=torch.int8, device="cuda"), torch.rand(C, device="cuda"))
    b.gspc_matmul_i8(a, w, out=y)
    assert torch.equal(y, b.gspc_matmul_i8(a, w))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_workspace_is_as_large_as_said(gpu, shape, kind):
    """What a workspace held before does not matter, and a call given as many bytes as it asks for leaves what lies behind them."""
    torch, b = gpu
    N, P, C, groups = shape
    x, gamma, beta = norm_inputs(N, P, C, 11)
    x, gamma, beta = dev(torch, x, getattr(torch, kind)), dev(torch, gamma), dev(torch, beta)
    dtype = b.GSPC_F32 if kind == "float32" else b.GSPC_BF16

    def scratch(need):
        whole = torch.full((need // 4 + 64,), float("nan"), device="cuda")
        whole[need // 4:] = 7.0
        return whole, whole[:need // 4]

    def run(forward, rows8, backward, backward8):
        st = torch.empty(N, groups, 2, device="cuda")
        y = b.gspc_group_norm(x, gamma, beta, groups, act=b.ACT_SILU, stats=st, workspace=forward)
        q = b.gspc_group_norm(x, gamma, beta, groups, act=b.ACT_SILU, dtype=b.GSPC_I8, workspace=rows8)
        kept = b.gspc_quantize_rows(x)
        return (y, st, *q, *b.gspc_group_norm_backward(y, x, st, gamma, beta, groups, b.ACT_SILU, workspace=backward),
                *b.gspc_group_norm_backward(y, kept, st, gamma, beta, groups, b.ACT_SILU, workspace=backward8))

    needs = [b.gspc_group_norm_workspace_bytes(N, P, C, groups, dtype), b.gspc_group_norm_workspace_bytes(N, P, C, groups, dtype, True),
             b.gspc_group_norm_backward_workspace_bytes(N, P, C, groups, dtype, dtype),
             b.gspc_group_norm_backward_workspace_bytes(N, P, C, groups, dtype, b.GSPC_I8)]
    assert all(n % 4 == 0 for n in needs)
    spaces = [scratch(n) for n in needs]
    got = run(*(view for _, view in spaces))
    assert all(bool((whole[n // 4:] == 7.0).all()) for (whole, _), n in zip(spaces, needs))
    assert all(bool(t.isfinite().all()) for t in got)
    assert all(torch.equal(p, q) for p, q in zip(got, run(None, None, None, None)))


def test_tensors_past_32_bits(gpu):
    """Contiguous tensors of more than 2^32 elements: the same 2048 images over and over.  The first and the last ones get, bit by
    bit, what these images get by themselves (2048 fill the chip, so that sums are taken in the same order)."""
    torch, b = gpu
    P, C, some = 64, 128, 2048
    N = (1 << 32) // (P * C) + some                             # 2^32 and 2048 images more
    small = torch.randn(some, P, C, device="cuda").bfloat16()
    x = small.repeat(N // some, 1, 1)
    assert N % some == 0 and x.numel() > 1 << 32

    def check(big, want):
        n = want.shape[0]
        assert torch.equal(big[:n], want) and torch.equal(big[-n:], want)

    out = torch.empty_like(x)
    b.gspc_pack_channels_last(x, out=out.view(N, C, P))         # (planes of 64 channels as tokens)
    check(out.view(N, C, P), b.gspc_pack_channels_last(small))
    gamma, beta = 1 + 0.1 * torch.randn(C, device="cuda"), 0.1 * torch.randn(C, device="cuda")
    st, some_st = torch.empty(N, 8, 2, device="cuda"), torch.empty(some, 8, 2, device="cuda")
    b.gspc_group_norm(x, gamma, beta, 8, act=b.ACT_SILU, out=out, stats=st)
    check(out, b.gspc_group_norm(small, gamma, beta, 8, act=b.ACT_SILU, stats=some_st))
    check(st, some_st)
    b.gspc_group_norm_backward(x, x, st, gamma, beta, 8, b.ACT_SILU, dx=out)
    check(out, b.gspc_group_norm_backward(small, small, some_st, gamma, beta, 8, b.ACT_SILU)[0])
    q = b.gspc_group_norm(x, gamma, beta, 8, act=b.ACT_SILU, dtype=b.GSPC_I8)
    some_q = b.gspc_group_norm(small, gamma, beta, 8, act=b.ACT_SILU, dtype=b.GSPC_I8)
    for t, want in zip(q, some_q):
        check(t, want)
    w = b.gspc_quantize_rows(torch.randn(C, C, device="cuda"))
    b.gspc_matmul_i8(q, w, out=out)
    check(out.view(N * P, C), b.gspc_matmul_i8(some_q, w))
    b.gspc_dequantize_rows(q, C, out=out)
    tokens = b.gspc_dequantize_rows(some_q, C, dtype=b.GSPC_BF16)
    check(out.view(N * P, C), tokens)
    for t, want in zip(b.gspc_quantize_rows(out), b.gspc_quantize_rows(tokens)):
        check(t, want)
