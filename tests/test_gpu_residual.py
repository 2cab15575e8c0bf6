"""The norms of a residual block with its gate, dropout and residual on the GPU, forward and gradient, against their definition in 64 bits
(block_reference says what errors are allowed and why)."""
import itertools

import numpy as np
import pytest

from block_reference import B, U, act64, backward64, dropout_factors, f8_read, forward64, normalise, on_side_stream
from test_gpu_parity import gpu  # noqa: F401  (fixture)
from test_gpu_tokens import dev, host, strided

pytestmark = pytest.mark.gpu
NAMES = ("gate", "post_gamma", "post_beta", "pre_gamma", "pre_beta")


def setting(rng, rows, C, post, pre, gates, act, scale, drop, beta=True):
    """(arguments of the calls with numpy parameters, the definition's)"""
    p = {"post": post, "pre": pre, "act": act, "scale": scale, "drop": drop, "seed": int(rng.integers(1 << 62)), "offset": int(rng.integers(1 << 40))}
    for k, kind in (("post", post), ("pre", pre)):
        p[k + "_gamma"] = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32) if kind else None
        p[k + "_beta"] = (0.2 * rng.standard_normal(C)).astype(np.float32) if kind and beta else None
    p["gate"] = (0.5 + 0.3 * rng.standard_normal((gates, C))).astype(np.float32) if gates else None
    q = {k: (None if v is None else v.astype(float)) if k in NAMES else v for k, v in p.items()}
    q.update(mask=dropout_factors(rows, C, drop, p["seed"], p["offset"]) if drop else None, eps=1e-5)
    return p, q


def on_gpu(torch, p):
    return {k: dev(torch, v) if isinstance(v, np.ndarray) else v for k, v in p.items()}


def inputs(rng, rows, C):
    x = rng.standard_normal((rows, C)) * np.exp(0.5 * rng.standard_normal(C)) + 0.5 * rng.standard_normal(C)
    return x.astype(np.float32)


SIZES = [(1, 1), (5, 2), (3, 7), (130, 8), (7, 9), (20, 16), (33, 60), (4, 63), (300, 64), (10, 65), (6, 100), (9, 128), (12, 130), (50, 333),
         (3, 512), (2, 513), (1, 1000), (30, 1024), (2, 1025), (3, 2048), (4, 2056), (1, 4096), (3, 5003), (2, 8192), (5000, 24), (2100, 520)]
TYPES = ["float32", "bfloat16"]


def gates_of(rows, k):
    """None, one, one for each token, or some number in between."""
    return (None, 1, rows, next(d for d in (4, 3, 2, 5, 7, 1) if rows % d == 0))[k % 4]


def cases():
    for k, (rows, C) in enumerate(SIZES):
        for j, (tx, th) in enumerate(itertools.product(TYPES, TYPES)):
            n = 5 * k + 3 * j
            yield rows, C, n % 3, 1 + (n // 3 + j) % 2, gates_of(rows, n), (n // 2) % 3, (1.0, 0.5)[n % 2], (0.0, 0.25)[(n + j) // 2 % 2], tx, th


@pytest.mark.parametrize("case", list(cases()), ids=str)
def test_forward(gpu, case):
    torch, b = gpu
    rows, C, post, pre, gates, act, scale, drop, tx, th = case
    rng = np.random.default_rng(rows * 10000 + C)
    p, q = setting(rng, rows, C, post, pre, gates, act, scale, drop, beta=C % 2 == 0)
    x, h = dev(torch, inputs(rng, rows, C), getattr(torch, tx)), dev(torch, inputs(rng, rows, C), getattr(torch, th))
    p, want = on_gpu(torch, p), forward64(q, host(x), host(h))
    stats = torch.full((rows + 1, 4), 9.0, device="cuda")
    xo, z = b.gspc_residual_norm(x, h, stats=stats[:-1], **p)
    assert xo.dtype == z.dtype == x.dtype and bool((stats[-1] == 9).all())
    for got, name, error in ((xo, "xo", "e_xo"), (z, "z", "e_z")):
        w = want[name]
        tol = want[error] + (B if tx == "bfloat16" else U) * np.abs(w) * 1.01 + 1e-30
        assert (np.abs(host(got) - w) <= tol).all(), (name, np.max(np.abs(host(got) - w) / tol))
    got, w = host(stats[:-1]), want["stats"]
    for k, err in ((0, 256 * U * (1 / w[:, 1] + np.abs(w[:, 0]))), (2, 256 * U * (1 / w[:, 3] + np.abs(w[:, 2])) + want["far"][:, 0])):
        assert (np.abs(got[:, k] - w[:, k]) <= err).all()
        assert (np.abs(got[:, k + 1] / w[:, k + 1] - 1) <= 256 * U * (1 + np.abs(w[:, k]) * w[:, k + 1]) + (w[:, 3] * want["far"][:, 0] * 2 if k else 0)).all()
    # rows with gaps, outputs among others, another type of z, the same bits; and in place
    (_, xs), (_, hs) = strided(torch, x, 10), strided(torch, h, 6)
    wide, zs = strided(torch, torch.zeros_like(x), 6)
    wide_xo, xos = strided(torch, torch.zeros_like(x), 6)
    b.gspc_residual_norm(xs, hs, xo=xos, out=zs, **p)
    assert torch.equal(xos, xo) and torch.equal(zs, z)
    for t in (wide, wide_xo):
        assert bool(t[..., :3].isnan().all()) and bool(t[..., -3:].isnan().all())
    other = torch.float32 if tx == "bfloat16" else torch.bfloat16
    z2 = b.gspc_residual_norm(x, h, out=torch.empty_like(x, dtype=other), **p)[1]
    assert torch.equal(z2.bfloat16(), z.bfloat16())
    mine = x.clone()
    got = b.gspc_residual_norm(mine, h, xo=mine, out=torch.empty_like(z), **p)
    assert got[0] is mine and torch.equal(mine, xo) and torch.equal(got[1], z)
    # without a second norm, and 8-bit float rows of z: within half a step of it, and what is rounded to them twice
    only = {k: v for k, v in p.items() if not k.startswith("pre") and k != "act"}
    alone, none = b.gspc_residual_norm(x, h, **only)
    assert none is None and torch.equal(alone, xo)
    z32 = z if tx == "float32" else z2
    q8, s8 = b.gspc_residual_norm(x, h, dtype=b.GSPC_F8, **p)[1]
    want8 = b.gspc_quantize_rows_f8(z32)
    assert torch.equal(q8.view(torch.uint8), want8[0].view(torch.uint8)) and torch.equal(s8, want8[1])


# a team's lanes are more than a token's channels, which no parameter says
UNEVEN = [(7, 3), (7, 24), (60, 37), (7, 40), (5, 65), (9, 133), (3, 520), (3, 1000), (2, 1544), (2, 4104), (2, 5003)]


@pytest.mark.parametrize("rows,C", UNEVEN)
@pytest.mark.parametrize("post,pre", itertools.product((0, 1, 2), (1, 2)))
def test_norms_without_parameters(gpu, rows, C, post, pre):
    """Forward and gradient, whose sums have zeros where a lane has no channel."""
    torch, b = gpu
    rng = np.random.default_rng(rows * 1000 + C)
    p = {"post": post, "pre": pre, "act": 0, "scale": 1.0, "drop": 0.0}
    q = {**p, **dict.fromkeys(NAMES), "mask": None, "eps": 1e-5}
    x, h, dz, dxo = (dev(torch, inputs(rng, rows, C) + np.float32(k)) for k in (1, 3, 0, 0))
    stats = torch.empty(rows, 4, device="cuda")
    xo, z = b.gspc_residual_norm(x, h, stats=stats, **p)
    want = forward64(q, host(x), host(h))
    for got, name, error in ((xo, "xo", "e_xo"), (z, "z", "e_z")):
        assert (np.abs(host(got) - want[name]) <= want[error] + U * np.abs(want[name]) * 1.01 + 1e-30).all(), name
    q8, s8 = b.gspc_residual_norm(x, h, dtype=b.GSPC_F8, **p)[1]
    want8 = b.gspc_quantize_rows_f8(z)
    assert torch.equal(q8.view(torch.uint8), want8[0].view(torch.uint8)) and torch.equal(s8, want8[1])
    got = b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, **p)
    check_grads(torch, got, backward64(q, host(dz), host(dxo), host(xo), host(h), host(stats)), {})


@pytest.mark.parametrize("rows,C", [(1, 1), (7, 60), (130, 130), (3, 1000), (2, 8192)])
@pytest.mark.parametrize("kind", [1, 2])
def test_norm_alone(gpu, rows, C, kind):
    """Without h: a token norm, of what a network's first block reads."""
    torch, b = gpu
    rng = np.random.default_rng(rows + C)
    x, g = dev(torch, inputs(rng, rows, C) + np.float32(3)), dev(torch, rng.standard_normal(C).astype(np.float32))
    same, z = b.gspc_residual_norm(x, pre=kind, pre_gamma=g, act=b.ACT_SILU)
    assert same is x
    xh, mean, rstd = normalise(host(x), kind, 1e-5)
    v = xh * host(g)
    tol = 1.1 * 256 * U * (1 + np.abs(xh) + np.abs(mean) * rstd) * np.abs(host(g)) + 16 * U * np.abs(v) + 1e-30
    assert (np.abs(host(z) - act64(v, 2)) <= tol).all()
    half, z2 = b.gspc_residual_norm(x, pre=kind, pre_gamma=g, act=b.ACT_SILU, scale=0.5)
    assert torch.equal(half, x * 0.5)
    assert torch.equal(z2, b.gspc_residual_norm(half, pre=kind, pre_gamma=g, act=b.ACT_SILU)[1])


def test_offsets_outliers_and_constant_tokens(gpu):
    """An offset far above the spread does not cancel in the variance; a constant token's is zero and its norm is the offset parameter."""
    torch, b = gpu
    for C in (60, 1000, 4100):
        rng = np.random.default_rng(C)
        x = inputs(rng, 6, C) + np.float32(1000)
        x[1, 0] = 3e4
        x[2] = 3.25
        beta = dev(torch, rng.standard_normal(C).astype(np.float32))
        z = host(b.gspc_residual_norm(dev(torch, x), pre=b.NORM_LAYER, pre_beta=beta)[1])
        xh, mean, rstd = normalise(x.astype(float), 2, 1e-5)
        assert np.array_equal(z[2], host(beta))
        tol = 256 * U * (1 + np.abs(xh) + np.abs(mean) * rstd) + 8 * U * np.abs(host(beta))
        keep = [0, 1, 3, 4, 5]
        assert (np.abs(z - xh - host(beta)) <= tol)[keep].all()


@pytest.mark.parametrize("C", [7, 24, 60, 512, 1000, 1100, 4100, 8192])
@pytest.mark.parametrize("kind", [1, 2])
def test_squares_past_fp32(gpu, C, kind):
    """Finite tokens whose mean square fp32 does not hold: 1 / deviation is 0, the norm's result its offset parameter, and gradients are numbers.  A constant
    token as large has no spread all the same."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(C)
    x, h = torch.randn(12, C, device="cuda", generator=g), torch.randn(12, C, device="cuda", generator=g)
    dz, dxo, beta = torch.randn(12, C, device="cuda", generator=g), torch.randn(12, C, device="cuda", generator=g), torch.randn(C, device="cuda", generator=g)
    gate, gamma = torch.full((C,), 0.5, device="cuda"), torch.full((C,), 1.5, device="cuda")
    kw = dict(gate=gate, post=kind, post_gamma=gamma, post_beta=beta, pre=kind, pre_gamma=gamma, pre_beta=beta)
    clean = b.gspc_residual_norm(x, h, **kw)
    h[3] *= 1e21
    x[8] *= 1e21
    x[8, 0] = h[3, 0] = 1e21                            # (one at least, of either norm)
    stats = torch.empty(12, 4, device="cuda")
    xo, z = b.gspc_residual_norm(x, h, stats=stats, **kw)
    keep = [r for r in range(12) if r not in (3, 8)]
    assert torch.equal(xo[keep], clean[0][keep]) and torch.equal(z[keep], clean[1][keep])
    assert stats[3, 1] == 0 and stats[8, 3] == 0
    assert torch.equal(xo[3], x[3] + 0.5 * beta) and torch.equal(z[8], beta)
    grads = b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, **kw)
    assert all(bool(t.isfinite().all()) for t in grads)
    assert torch.equal(grads.dx[8], dxo[8]) and bool((grads.dh[3] == 0).all())
    x[5] = 2.0 ** 70
    z = b.gspc_residual_norm(x, pre=kind, pre_beta=beta)[1]
    assert torch.equal(z[5], beta) and bool(z.isfinite().all())


@pytest.mark.parametrize("C", [60, 1024, 4100])
def test_what_is_not_finite_stays_in_its_token(gpu, C):
    torch, b = gpu
    rng = np.random.default_rng(C)
    rows = 40
    p, _ = setting(rng, rows, C, 2, 1, 4, 2, 1.0, 0.25)
    p = on_gpu(torch, p)
    x, h = (dev(torch, inputs(rng, rows, C)) for _ in range(2))
    clean = b.gspc_residual_norm(x, h, **p)
    h[3, 5], x[17, C - 1] = float("nan"), float("inf")
    xo, z = b.gspc_residual_norm(x, h, **p)
    keep = [r for r in range(rows) if r not in (3, 17)]
    assert torch.equal(xo[keep], clean[0][keep]) and torch.equal(z[keep], clean[1][keep])
    assert bool(z[3].isnan().all()) and xo[17, C - 1] == float("inf") and bool(xo[17, :C - 1].isfinite().all())
    m = torch.from_numpy(dropout_factors(rows, C, 0.25, p["seed"], p["offset"])).cuda()
    assert torch.equal(xo[3][m[3] == 0], x[3][m[3] == 0])       # where the block's output is dropped the stream goes on


@pytest.mark.parametrize("C", [3, 24, 37, 130, 520, 4104])
def test_tokens_that_are_no_number_as_8_bit_float_rows_and_back(gpu, C):
    """What lies past their last column is zero all the same, and in the gradient they have no say in other tokens."""
    torch, b = gpu
    rng = np.random.default_rng(C)
    x, h, dz, dxo = (dev(torch, inputs(rng, 9, C)) for _ in range(4))
    h[3, C - 1], x[6, 0] = float("nan"), float("inf")
    p = {"post": 2, "pre": 2, "act": 2}
    stats = torch.empty(9, 4, device="cuda")
    xo, z = b.gspc_residual_norm(x, h, stats=stats, **p)
    q8, s8 = b.gspc_residual_norm(x, h, dtype=b.GSPC_F8, **p)[1]
    want = b.gspc_quantize_rows_f8(z)
    assert torch.equal(q8.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s8, want[1])
    assert not bool(q8[:, C:].view(torch.uint8).any()) and bool(q8[3, :C].float().isnan().all())
    got = b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, **p)
    keep = [0, 1, 2, 4, 5, 7, 8]
    less = b.gspc_residual_norm_backward(*(t[keep].contiguous() for t in (dz, dxo, xo, h, stats)), **p)
    assert torch.equal(got.dx[keep], less.dx) and torch.equal(got.dh[keep], less.dh) and bool(less.dx.isfinite().all())


# ---- the gradient ------------------------------------------------------------------------------------------
def check_grads(torch, got, want, types):
    for name, (w, size) in want.items():
        g = getattr(got, name)
        if g is None:
            continue
        half = B if types.get(name) == "bfloat16" else U
        tol = 256 * U * size + half * np.abs(w) * 1.01 + 1e-30
        err = np.abs(host(g).reshape(w.shape) - w)
        assert (err <= tol).all(), (name, np.max(err / tol))


@pytest.mark.parametrize("case", list(cases()), ids=str)
def test_backward(gpu, case):
    torch, b = gpu
    rows, C, post, pre, gates, act, scale, drop, tx, th = case
    act = 2 if act == 1 else act                                # (ReLU's jump: below, where no value is near it)
    rng = np.random.default_rng(rows * 10000 + C + 1)
    p, q = setting(rng, rows, C, post, pre, gates, act, scale, drop, beta=C % 2 == 0)
    p = on_gpu(torch, p)
    x, h, dz, dxo = (dev(torch, inputs(rng, rows, C), getattr(torch, t)) for t in (tx, th, th, tx))
    stats = torch.empty(rows, 4, device="cuda")
    xo, _ = b.gspc_residual_norm(x, h, stats=stats, **p)
    run = lambda *a, **k: b.gspc_residual_norm_backward(*a, **{**p, **k})  # noqa: E731
    got = run(dz, dxo, xo, h, stats)
    want = backward64(q, host(dz), host(dxo), host(xo), host(h), host(stats))
    types = {"dx": tx, "dh": th}
    check_grads(torch, got, want, types)
    assert got.dx.dtype == x.dtype and got.dh.dtype == h.dtype
    for name in NAMES:
        assert (getattr(got, "d" + name) is None) == (p[name] is None)
    # rows with gaps, given outputs, in place: the same bits
    gap = [strided(torch, t, 6)[1] for t in (dz, dxo, xo, h)]
    wide, dxs = strided(torch, torch.zeros_like(x), 6)
    outs = {"d" + k: torch.full_like(p[k], float("nan")) for k in NAMES if p[k] is not None}
    two = run(*gap, stats, dx=dxs, dh=torch.empty_like(h), **outs)
    mine, own = dxo.clone(), h.clone()
    three = run(dz, mine, xo, own, stats, dx=mine, dh=own)
    assert bool(wide[..., :3].isnan().all()) and bool(wide[..., -3:].isnan().all())
    for name, g in got._asdict().items():
        if g is not None:
            assert torch.equal(g, getattr(two, name).view(g.shape)) and torch.equal(g, getattr(three, name)), name
    # either gradient alone
    check_grads(torch, run(dz, None, xo, h, stats), backward64(q, host(dz), None, host(xo), host(h), host(stats)), types)
    check_grads(torch, run(None, dxo, xo, h, stats), backward64(q, None, host(dxo), host(xo), host(h), host(stats)), types)


def test_backward_of_a_norm_alone(gpu):
    torch, b = gpu
    rng = np.random.default_rng(3)
    for rows, C, kind in ((1, 5, 2), (40, 100, 1), (700, 512, 2)):
        p, q = setting(rng, rows, C, 0, kind, None, 2, 0.5, 0.0)
        p = on_gpu(torch, p)
        x, dz, dxo = (dev(torch, inputs(rng, rows, C)) for _ in range(3))
        stats = torch.empty(rows, 4, device="cuda")
        xo, _ = b.gspc_residual_norm(x, stats=stats, **p)
        got = b.gspc_residual_norm_backward(dz, dxo, xo, None, stats, **p)
        assert got.dh is None and got.dgate is None
        check_grads(torch, got, backward64(q, host(dz), host(dxo), host(xo), None, host(stats)), {})


def test_backward_through_relu_away_from_its_jump(gpu):
    torch, b = gpu
    rng = np.random.default_rng(4)
    rows, C = 60, 130
    p, q = setting(rng, rows, C, 1, 2, 1, 1, 1.0, 0.0)
    p["pre_beta"] = np.where(np.arange(C) % 2, 40, -40).astype(np.float32)      # |xh gamma| is at most sqrt(130) times 1.8
    q["pre_beta"] = p["pre_beta"].astype(float)
    p = on_gpu(torch, p)
    x, h, dz, dxo = (dev(torch, inputs(rng, rows, C)) for _ in range(4))
    stats = torch.empty(rows, 4, device="cuda")
    xo, z = b.gspc_residual_norm(x, h, stats=stats, **p)
    assert bool((z[:, ::2] == 0).all()) and bool((z[:, 1::2] > 0).all())
    check_grads(torch, b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, **p), backward64(q, host(dz), host(dxo), host(xo), host(h), host(stats)), {})


@pytest.mark.parametrize("post,pre,act,gates", [(2, 2, 2, 2), (1, 1, 2, 1), (0, 2, 0, 6), (2, 1, 0, None)])
def test_gradient_against_differences(gpu, post, pre, act, gates):
    """Central differences of the definition in 64 bits along each input (step 1e-5: its third derivative leaves 1e-10 times a constant of the order
    of the tokens' inverse deviations cubed; rounding 1e-16 / 1e-5), and the gradient in fp32: 1e-4 of the sum of magnitudes covers both."""
    torch, b = gpu
    rng = np.random.default_rng(5 + post)
    rows, C = 6, 20
    p, q = setting(rng, rows, C, post, pre, gates, act, 0.7, 0.25)
    x, h, dz, dxo = (inputs(rng, rows, C) for _ in range(4))
    d = on_gpu(torch, p)
    stats = torch.empty(rows, 4, device="cuda")
    xo, _ = b.gspc_residual_norm(dev(torch, x), dev(torch, h), stats=stats, **d)
    got = b.gspc_residual_norm_backward(dev(torch, dz), dev(torch, dxo), xo, dev(torch, h), stats, **d)

    def loss(name, direction, step):
        q2, x2, h2 = dict(q), x.astype(float), h.astype(float)
        if name == "x":
            x2 = x2 + step * direction
        elif name == "h":
            h2 = h2 + step * direction
        else:
            q2[name] = q[name] + step * direction
        out = forward64(q2, x2, h2)
        return (out["z"] * dz).sum() + (out["xo"] * dxo).sum()

    for name in ("x", "h") + tuple(k for k in NAMES if q[k] is not None):
        grad = host(getattr(got, "d" + name))
        for _ in range(4):
            direction = rng.standard_normal(grad.shape)
            want = (loss(name, direction, 1e-5) - loss(name, direction, -1e-5)) / 2e-5
            assert abs((grad * direction).sum() - want) <= 1e-4 * np.abs(grad * direction).sum(), name


@pytest.mark.parametrize("rows,C,gates", [(1, 8, 1), (5000, 24, 5000), (2100, 520, 3), (300, 1024, 1), (2100, 5003, 2100), (70000, 64, 1)])
def test_workspace_is_as_large_as_said(gpu, rows, C, gates):
    torch, b = gpu
    rng = np.random.default_rng(rows)
    p, _ = setting(rng, rows, C, 2, 2, gates, 2, 1.0, 0.1)
    p = on_gpu(torch, p)
    x, h, dz, dxo = (torch.randn(rows, C, device="cuda").bfloat16() for _ in range(4))
    stats = torch.empty(rows, 4, device="cuda")
    xo, _ = b.gspc_residual_norm(x, h, stats=stats, **p)
    need = b.gspc_residual_norm_backward_workspace_bytes(rows, C, gates)
    whole = torch.full((need // 4 + 64,), float("nan"), device="cuda")
    whole[need // 4:] = 7.0
    got = b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, workspace=whole[:need // 4], **p)
    assert bool((whole[need // 4:] == 7.0).all())
    for g, w in zip(got, b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, **p)):
        assert bool(g.isfinite().all()) and torch.equal(g, w)
    with pytest.raises(b.GspcError, match="SPACE"):
        b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, workspace=whole[:need // 4 - 1], **p)


def test_many_tokens_sum_well(gpu):
    """Parameters' gradients over a million tokens of ones: whole numbers that fp32 sums in chains of a million would lose."""
    torch, b = gpu
    rows, C = 1 << 20, 64
    one = torch.ones(C, device="cuda")
    xo, h = torch.zeros(rows, C, device="cuda"), torch.ones(rows, C, device="cuda")
    stats = torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda").repeat(rows, 1)
    dz = torch.full((rows, C), 1 + 2.0 ** -10, device="cuda")
    got = b.gspc_residual_norm_backward(dz, xo, xo, h, stats, gate=one, pre=b.NORM_RMS, pre_beta=one)
    want = rows * (1 + 2.0 ** -10)              # exact in fp32
    assert bool((got.dpre_beta == want).all()) and bool((got.dgate == want).all())


def test_no_tokens(gpu):
    torch, b = gpu
    x, h = torch.zeros(0, 40, device="cuda"), torch.zeros(0, 40, device="cuda")
    g = torch.ones(40, device="cuda")
    kw = dict(gate=torch.ones(3, 40, device="cuda"), post=2, post_gamma=g, pre=1, pre_gamma=g)
    xo, z = b.gspc_residual_norm(x, h, **kw)
    assert xo.shape == z.shape == (0, 40)
    got = b.gspc_residual_norm_backward(z, xo, xo, h, torch.zeros(0, 4, device="cuda"), dgate=torch.full((3, 40), 5.0, device="cuda"), **kw)
    assert got.dx.shape == (0, 40)
    for t in (got.dgate, got.dpost_gamma, got.dpre_gamma):
        assert bool((t == 0).all())


def step_of_a_block(torch, b, x, h, dz, dxo, p, step):
    stats = torch.empty(x.shape[0], 4, device="cuda")
    xo, z = b.gspc_residual_norm(x, h, stats=stats, step=step, **p)
    return (xo, z, stats, *b.gspc_residual_norm_backward(dz, dxo, xo, h, stats, step=step, **p))


def test_side_stream_and_two_replayed_graphs(gpu):
    """Two graphs of the same block, with their own workspaces from torch's pools, replayed in turns with new inputs and masks, and eager calls between."""
    torch, b = gpu
    rows, C = 1200, 320
    rng = np.random.default_rng(8)
    p, _ = setting(rng, rows, C, 2, 1, 4, 2, 1.0, 0.3)
    p = on_gpu(torch, p)
    t = [torch.randn(rows, C, device="cuda").bfloat16() for _ in range(4)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    want = step_of_a_block(torch, b, *t, p, step)
    with on_side_stream(torch, b) as s:
        got = step_of_a_block(torch, b, *t, p, step)
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                graphs.append((graph, step_of_a_block(torch, b, *t, p, step)))
        for k in range(6):
            graph, held = graphs[k % 2]
            for x in t:
                x.copy_(torch.randn_like(x))
            step.fill_(k)
            graph.replay()
            want = step_of_a_block(torch, b, *t, p, step)
            s.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(held, want)), k


def test_tokens_past_32_bits(gpu):
    """More than 2^32 elements: the first and the last tokens get, bit by bit, what they get by themselves."""
    torch, b = gpu
    C, some = 512, 2048
    rows = (1 << 32) // C + some
    small = torch.randn(some, C, device="cuda").bfloat16()
    x = small.repeat(rows // some, 1)
    gamma = 1 + 0.1 * torch.randn(C, device="cuda")
    kw = dict(post=b.NORM_LAYER, post_gamma=gamma, pre=b.NORM_RMS, pre_gamma=gamma)
    stats, some_stats = torch.empty(rows, 4, device="cuda"), torch.empty(some, 4, device="cuda")
    xo, z = b.gspc_residual_norm(x, x, stats=stats, **kw)
    want = b.gspc_residual_norm(small, small, stats=some_stats, **kw)
    for big, w in ((xo, want[0]), (z, want[1]), (stats, some_stats)):
        assert torch.equal(big[:some], w) and torch.equal(big[-some:], w)
    got = b.gspc_residual_norm_backward(z, x, xo, x, stats, **kw)
    want = b.gspc_residual_norm_backward(want[1], small, want[0], small, some_stats, **kw)
    for big, w in ((got.dx, want.dx), (got.dh, want.dh)):
        assert torch.equal(big[:some], w) and torch.equal(big[-some:], w)


def test_8_bit_float_rows_leave_what_lies_behind(gpu):
    torch, b = gpu
    for rows, C in ((3, 5), (33, 60), (20, 130), (2, 1025)):
        x = torch.randn(rows, C, device="cuda")
        q = torch.full((rows + 2, b.gspc_f8_pitch(C)), 1.5, device="cuda").to(torch.float8_e4m3fn)
        s = torch.full((rows + 2, b.gspc_f8_scale_pitch(C)), 77, dtype=torch.uint8, device="cuda")
        b.gspc_residual_norm(x, pre=b.NORM_LAYER, out=(q[1:-1], s[1:-1]))
        assert bool((q.float()[[0, -1]] == 1.5).all()) and bool((s[[0, -1]] == 77).all())
        z = b.gspc_residual_norm(x, pre=b.NORM_LAYER)[1]
        back = f8_read(q[1:-1].float().double().cpu().numpy(), s[1:-1].cpu().numpy())
        assert (back[:, C:] == 0).all() and (np.abs(back[:, :C] - host(z)) <= np.maximum(2.0 ** -4 * np.abs(host(z)), 2.0 ** -10 * np.abs(host(z)).max(1, keepdims=True))).all()
