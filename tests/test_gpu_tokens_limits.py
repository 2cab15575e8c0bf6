"""Channels-last operators at counts that pass what one launch may have: many small images, one very large plane."""
import pytest

from test_gpu_parity import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
MANY = 17_000_000               # images: in blocks of 256 threads more than 2^32 threads


@pytest.mark.parametrize("C,P", [(8, 8), (3, 2)])
def test_layout_of_many_images(gpu, C, P):
    torch, b = gpu
    x = torch.randn(MANY, C, P, device="cuda").bfloat16()
    y = b.gspc_pack_channels_last(x)
    assert torch.equal(y, x.transpose(1, 2))
    z = b.gspc_unpack_channels_last(y, dtype=b.GSPC_BF16)
    assert torch.equal(z, x)


def test_layout_of_one_large_plane(gpu):
    """2^24 + 1 tiles of one plane: a number made of its place in each of its elements."""
    torch, b = gpu
    C, P, piece = 8, (1 << 30) + 1, 1 << 26
    x = torch.empty(1, C, P, dtype=torch.int16, device="cuda")
    number = lambda c, at: ((torch.arange(at, min(at + piece, P), device="cuda") * 40503 + c * 977) & 0x3fff).short()  # noqa: E731
    for c in range(C):
        for at in range(0, P, piece):
            x[0, c, at:at + piece] = number(c, at)
    y = b.gspc_pack_channels_last(x.view(torch.bfloat16)).view(torch.int16)
    for c in range(C):
        for at in range(0, P, piece):
            assert torch.equal(y[0, at:at + piece, c], number(c, at)), (c, at)


def pieces(call, *tensors):
    """What `call` gives for four million images at a time (the last of them end with the tensors): too many for a block to hold each,
    as all of them are, so that sums are taken in the same order."""
    N, step = tensors[0].shape[0], 4_000_000
    for at in range(0, N, step):
        at = min(at, N - step)
        yield slice(at, at + step), call(*(t[at:at + step] for t in tensors))


@pytest.mark.parametrize("N,P,C", [(MANY, 1, 16), (9_600_000, 64, 7)])
def test_norm_of_many_images(gpu, N, P, C):
    """Every image gets, bit by bit, what it gets among fewer."""
    torch, b = gpu
    x = torch.randn(N, P, C, device="cuda", dtype=torch.bfloat16)
    gamma, beta = 1 + 0.1 * torch.randn(C, device="cuda"), 0.1 * torch.randn(C, device="cuda")
    norm = lambda t, **k: b.gspc_group_norm(t, gamma, beta, 1, act=b.ACT_SILU, **k)  # noqa: E731
    st = torch.empty(N, 1, 2, device="cuda")
    y = norm(x, stats=st)
    for at, want in pieces(norm, x):
        assert torch.equal(y[at], want)
    back = lambda d, t, s: b.gspc_group_norm_backward(d, t, s, gamma, beta, 1, b.ACT_SILU)  # noqa: E731
    dx = back(x, x, st)[0]
    for at, want in pieces(back, x, x, st):
        assert torch.equal(dx[at], want[0])
    del dx, y, want
    saved = lambda n: (torch.empty(n, 16, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"))  # noqa: E731
    kept = saved(N * P)
    q = norm(x, dtype=b.GSPC_I8, saved=kept)
    for at, want in pieces(lambda t: norm(t, dtype=b.GSPC_I8), x):
        rows = slice(at.start * P, at.stop * P)
        assert torch.equal(q[0][rows], want[0]) and torch.equal(q[1][rows], want[1])
        for got, codes in zip(kept, b.gspc_quantize_rows(x[at])):
            assert torch.equal(got[rows], codes)


@pytest.mark.parametrize("N,P,C", [(MANY, 1, 16), (3_000_000, 1, 9), (200_000, 65, 24)])
def test_parameter_gradients_of_many_images(gpu, N, P, C):
    """Against sums in 64 bits, which images' own sums enter without another rounding: 256 u of the sum of magnitudes, as for one image."""
    torch, b = gpu
    x = torch.randn(N, P, C, device="cuda", dtype=torch.bfloat16)
    gamma, beta = 1 + 0.1 * torch.randn(C, device="cuda"), 0.1 * torch.randn(C, device="cuda")
    st = torch.empty(N, 1, 2, device="cuda")
    b.gspc_group_norm(x, gamma, beta, 1, stats=st)
    _, dgamma, dbeta = b.gspc_group_norm_backward(x, x, st, gamma, beta, 1, b.ACT_SILU)
    sums, sizes = torch.zeros(2, C, dtype=torch.float64, device="cuda"), torch.zeros(2, C, dtype=torch.float64, device="cuda")
    for at in range(0, N, 1_000_000):
        at = slice(at, at + 1_000_000)
        xh = (x[at].double() - st[at][..., :1]) * st[at][..., 1:]
        z = xh * gamma + beta
        dz = x[at].double() * (torch.sigmoid(z) * (1 + z * (1 - torch.sigmoid(z))))
        for k, t in enumerate((dz * xh, dz)):
            sums[k] += t.sum((0, 1))
            sizes[k] += t.abs().sum((0, 1))
    shift = float((st[..., 0] * st[..., 1]).abs().max())
    off = (torch.stack((dgamma, dbeta)) - sums).abs() / (256 * 2.0 ** -24 * (1 + shift) * sizes)
    assert bool((off <= 1).all()), off.max()


@pytest.mark.parametrize("M,N", [(1, 20), (40, 40)])
@pytest.mark.parametrize("given", [False, True])
def test_longest_rows_through_the_binding(gpu, M, N, given):
    torch, b = gpu
    K = 133144
    a, w = b.gspc_quantize_rows(torch.ones(M, K, device="cuda")), b.gspc_quantize_rows(-torch.ones(N, K, device="cuda"))
    a[1].fill_(1.0)
    w[1].fill_(1.0)
    out = b.gspc_matmul_i8(a, w, out=torch.empty(M, N, device="cuda") if given else None, dtype=b.GSPC_F32, cols=K)
    assert bool((out == float(torch.tensor(-127.0 * 127 * K))).all())
    with pytest.raises(b.GspcError, match="133144"):
        b.gspc_matmul_i8(a, w, dtype=b.GSPC_F32)


@pytest.mark.parametrize("M,N,K", [(1, 50257, 272), (16, 41000, 128), (1, 128256, 80), (40, 33000, 272), (100, 50257, 144), (50000, 10, 80), (50000, 100, 272)])
def test_products_long_in_one_direction(gpu, M, N, K):
    """Few tokens and many filters, or the reverse: the integer sums, exact in fp32 (127 * 127 * 272 < 2^24)."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    q = lambda rows: torch.randint(-127, 128, (rows, K), dtype=torch.int8, device="cuda", generator=g)  # noqa: E731
    a, w = (q(M), torch.ones(M, device="cuda")), (q(N), torch.ones(N, device="cuda"))
    out = torch.full((M + 2, N + 5), 7.0, device="cuda")
    b.gspc_matmul_i8(a, w, out=out[1:-1, 2:-3])
    want = a[0].float() @ w[0].float().t().contiguous()         # (sums of whole numbers below 2^24: exact in any order)
    assert torch.equal(out[1:-1, 2:-3], want), b.gspc_last_kernel()
    assert bool((out[0] == 7).all() and (out[-1] == 7).all() and (out[:, :2] == 7).all() and (out[:, -3:] == 7).all())


def test_product_of_as_many_tokens_as_there_are(gpu):
    """2^31 - 1 tokens: more blocks than one launch may have.  Whole numbers, exact."""
    torch, b = gpu
    M, N, K, step = 0x7fffffff, 2, 16, 1 << 26
    a = (torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda"))
    w = (torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda"))
    out = b.gspc_matmul_i8(a, w, dtype=b.GSPC_F32)
    for at in range(0, M, step):
        assert torch.equal(out[at:at + step], a[0][at:at + step].float() @ w[0].float().t().contiguous()), at


@pytest.mark.parametrize("N,P,C,groups", [(3, 196, 48, 8), (2, 100, 60, 12), (5, 49, 96, 16), (1, 784, 24, 4), (2, 160, 35, 7)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradient_of_odd_groups_held(gpu, N, P, C, groups, dtype):
    """Groups of channels that are no multiple of four, x in fp32, three and four vectors a thread: as test_norm_backward, its tolerance."""
    import numpy as np
    from test_gpu_tokens import B, U, dev, grad64, host, norm_inputs
    torch, b = gpu
    x, gamma, beta = norm_inputs(N, P, C, N + 2 * P + C, offset=3.0)
    dy = dev(torch, np.random.default_rng(P).standard_normal((N, P, C)).astype(np.float32), getattr(torch, dtype))
    xd, gd, bd, st = dev(torch, x), dev(torch, gamma), dev(torch, beta), torch.empty(N, groups, 2, device="cuda")
    b.gspc_group_norm(xd, gd, bd, groups, act=b.ACT_SILU, stats=st)
    dx, dgamma, dbeta, size, size_g, size_b, xh, shift = grad64(host(dy), host(xd), host(st), gamma.astype(float), beta.astype(float), groups, 2)
    got = b.gspc_group_norm_backward(dy, xd, st, gd, bd, groups, b.ACT_SILU)
    tol = 256 * U * size * (1 + np.abs(xh) + np.abs(shift)) + (B * np.abs(dx) if dtype == "bfloat16" else 0) + 1e-30
    rel = 1 + np.abs(shift).max()
    assert (np.abs(host(got[0]) - dx) <= tol).all(), np.max(np.abs(host(got[0]) - dx) / tol)
    assert (np.abs(host(got[1]) - dgamma) <= 256 * U * rel * size_g + 1e-30).all()
    assert (np.abs(host(got[2]) - dbeta) <= 256 * U * rel * size_b + 1e-30).all()


def test_pairs_as_lists(gpu):
    torch, b = gpu
    x = torch.randn(2, 9, 24, device="cuda")
    pair = lambda: [torch.empty(18, 32, dtype=torch.int8, device="cuda"), torch.empty(18, device="cuda")]  # noqa: E731
    st, out, kept = torch.empty(2, 3, 2, device="cuda"), pair(), pair()
    assert b.gspc_group_norm(x, None, None, 3, out=out, stats=st, saved=kept) is out
    want = b.gspc_group_norm(x, None, None, 3, dtype=b.GSPC_I8)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    for p, q in zip(b.gspc_group_norm_backward(x, kept, st, None, None, 3), b.gspc_group_norm_backward(x, tuple(kept), st, None, None, 3)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("C", [1, 8])
def test_norm_of_one_image_as_long_as_there_are(gpu, C):
    """2^31 - 1 tokens: against 64 bits, piece by piece, with the tolerances of test_gpu_tokens (u = 2^-24, 2^-8 for a value rounded to bf16)."""
    torch, b = gpu
    P, step, U, B = 0x7fffffff, 1 << 25, 2.0 ** -24, 2.0 ** -8
    pieces = [slice(at, min(at + step, P)) for at in range(0, P, step)]
    x = torch.empty(1, P, C, dtype=torch.bfloat16, device="cuda")
    for s in pieces:
        x[0, s].normal_()
    x[0, -1] = 50.0                                             # (the last token counts, and is seen)
    gamma, beta = 1 + 0.1 * torch.randn(C, device="cuda"), 0.1 * torch.randn(C, device="cuda")
    st = torch.empty(1, 1, 2, device="cuda")
    y = b.gspc_group_norm(x, gamma, beta, 1, act=b.ACT_SILU, stats=st)
    mean = sum(float(x[0, s].double().sum()) for s in pieces) / (P * C)
    rstd = (sum(float((x[0, s].double() - mean).square().sum()) for s in pieces) / (P * C) + 1e-5) ** -0.5
    assert abs(float(st[0, 0, 0]) - mean) * rstd <= 256 * U and abs(float(st[0, 0, 1]) / rstd - 1) <= 256 * U
    rel = 1 + abs(mean) * rstd

    def expected(s, mean, rstd):
        xh = (x[0, s].double() - mean) * rstd
        z = xh * gamma + beta
        return xh, z, torch.sigmoid(z)
    for s in pieces:
        xh, z, sig = expected(s, mean, rstd)
        tol = 256 * U * (rel + xh.abs()) * (gamma.abs() + z.abs()) + 1e-30
        assert bool(((y[0, s].double() - z * sig).abs() <= tol + B * (z * sig).abs()).all()), s
    del y
    q, scale = b.gspc_group_norm(x, gamma, beta, 1, act=b.ACT_SILU, dtype=b.GSPC_I8)
    for s in pieces:
        xh, z, sig = expected(s, mean, rstd)
        want = z * sig
        tol = 256 * U * (rel + xh.abs()) * (gamma.abs() + z.abs()) + 1e-30
        err = (q[s, :C].double() * scale[s, None] - want).abs()
        assert bool((err <= 0.501 * want.abs().amax(1, keepdim=True) / 127 + 2 * tol + tol.amax(1, keepdim=True)).all()), s
        assert not bool(q[s, C:].any())
    del q, scale, want, err, tol
    dx, dgamma, dbeta = b.gspc_group_norm_backward(x, x, st, gamma, beta, 1, b.ACT_SILU)
    mean, rstd = (float(v) for v in st[0, 0])
    sums = torch.zeros(4, C, dtype=torch.float64, device="cuda")

    def slope(s):
        xh, z, sig = expected(s, mean, rstd)
        return xh, x[0, s].double() * sig * (1 + z * (1 - sig))
    for s in pieces:
        xh, dz = slope(s)
        sums += torch.stack(((dz * xh).sum(0), dz.sum(0), (dz * xh).abs().sum(0), dz.abs().sum(0)))
    assert bool(((dgamma - sums[0]).abs() <= 256 * U * rel * sums[2]).all()) and bool(((dbeta - sums[1]).abs() <= 256 * U * rel * sums[3]).all())
    A, BB, a_size, b_size = (float((t * g).sum()) / (P * C) for t, g in zip(sums[[1, 0, 3, 2]], (gamma, gamma, gamma.abs(), gamma.abs())))
    for s in pieces:
        xh, dz = slope(s)
        want = rstd * (gamma * dz - A - xh * BB)
        size = rstd * ((gamma * dz).abs() + a_size + xh.abs() * b_size)
        assert bool(((dx[0, s].double() - want).abs() <= 256 * U * size * (rel + xh.abs()) + B * want.abs() + 1e-30).all()), s


def test_layout_into_rows_of_tokens(gpu):
    torch, b = gpu
    x = torch.randn(2, 12, 35, device="cuda")
    for out in (torch.empty(70, 12, device="cuda"), torch.empty(2, 5, 7, 12, device="cuda")):
        assert b.gspc_pack_channels_last(x, out=out) is out and torch.equal(out.view(2, 35, 12), x.transpose(1, 2))
        assert b.gspc_pack_channels_last(x.view(2, 12, 5, 7), out=out.zero_()) is out and torch.equal(out.view(2, 35, 12), x.transpose(1, 2))
