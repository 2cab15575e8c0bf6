"""8-bit float rows and their products on the GPU against their definitions in 64 bits.

Tolerances.  Rows: none, codes and powers of two are whole numbers that have to be equal.  Products, with S = sum |a w| of an output and half a last
place (u = 2^-24, 2^-8 for bf16) of it for the output's own rounding:
  fp32 outputs: each of K additions cuts or rounds a partial sum of at most S at 2^-23 of it: K 2^-23 S, and the bias' u |y|;
  bf16 outputs: the same, and eight products are added with no bit below 2^-13 of the largest one's exponent: seven cut there, less than 2^-10 of
  the eight's sum of magnitudes: 2^-10 S."""
import numpy as np
import pytest

from block_reference import B, U, f8_read, f8_reference, on_side_stream
from test_gpu_parity import gpu  # noqa: F401  (fixture)
from test_gpu_tokens import dev, host, strided

pytestmark = pytest.mark.gpu


def values(torch, rows8):
    """(codes as float64 [rows, pitch], bytes) of a pair."""
    return rows8[0].float().double().cpu().numpy(), rows8[1].cpu().numpy()


def hard_rows(rng, rows, cols):
    x = (rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-12, 12, (rows, 1))).astype(np.float32)
    if rows > 100:
        x[3] = 0
        x[5] *= np.float32(1e-30)
        x[6] = np.float32(2.0 ** -149) * rng.integers(-3, 4, cols)     # the smallest numbers there are
        x[7] = np.float32(2.0 ** -127) * rng.integers(-3, 4, cols)
        x[8, -1] = np.inf
        x[9, 0] = np.nan
        x[10, :] = -np.inf
        x[11] = np.float32(3.4e38)
        x[12] = np.float32(448.0)                                      # the end of a power of two's range, and just behind it
        x[13] = np.nextafter(np.float32(448), np.float32(1000))
        x[14] = (np.arange(cols) % 61 - 30) / 4.0 + 1 / 32             # ties
        x[14, 0] = 256
        x[15] = np.float32(2.0) ** -(np.arange(cols) % 24)             # down through the smallest codes
        x[16] = np.float32(1.5 * 2.0 ** -10) * (np.arange(cols) % 3)
        x[16, 0] = 448
    return x


@pytest.mark.parametrize("cols", [1, 2, 7, 8, 9, 16, 60, 63, 64, 65, 120, 127, 128, 129, 130, 200, 255, 256, 333, 511, 512, 513, 640, 1001, 1500, 4104])
@pytest.mark.parametrize("rows", [1, 3, 127, 130, 389])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows(gpu, cols, rows, dtype):
    torch, b = gpu
    x = hard_rows(np.random.default_rng(cols * 1000 + rows), rows, cols)
    t = dev(torch, x, getattr(torch, dtype))
    x = t.float().cpu().numpy()
    _, view = strided(torch, t, 6)
    for src in (t, view):
        for which in (b.F8_ROWS, b.F8_COLUMNS, b.F8_BOTH):
            forms, outs = [], {}
            for bit, name, a in ((b.F8_ROWS, "out", x), (b.F8_COLUMNS, "out_t", x.T)):
                if which & bit:
                    n, pitch, s_pitch = len(a), b.gspc_f8_pitch(a.shape[1]), b.gspc_f8_scale_pitch(a.shape[1])
                    q = torch.full((n + 2, pitch), 1.5, device="cuda").to(torch.float8_e4m3fn)
                    # (the scales' first row begins on a word: s_pitch is a multiple of four)
                    s = torch.full((n + 2, s_pitch), 77, dtype=torch.uint8, device="cuda")
                    forms.append((a, q, s))
                    outs[name] = q[1:-1], s[1:-1]
            b.gspc_quantize_rows_f8(src, **outs)
            for a, q, s in forms:
                want, code = f8_reference(a)
                got = q.float().double().cpu().numpy()
                assert (got[0] == 1.5).all() and (got[-1] == 1.5).all() and (s[0] == 77).all() and (s[-1] == 77).all()
                assert np.array_equal(got[1:-1], want, equal_nan=True)
                assert np.array_equal(s[1:-1].cpu().numpy(), code)
                back = torch.full((a.shape[0], a.shape[1] + 6), 5.0, dtype=t.dtype, device="cuda")
                b.gspc_dequantize_rows_f8((q[1:-1], s[1:-1]), a.shape[1], out=back[:, 3:-3])
                want = torch.from_numpy(f8_read(want, code)[:, :a.shape[1]]).to(t.dtype)
                assert torch.equal(torch.nan_to_num(back[:, 3:-3].cpu(), nan=-1), torch.nan_to_num(want, nan=-1))
                assert (back[:, :3] == 5).all() and (back[:, -3:] == 5).all()


def test_rows_of_nothing_and_allocated(gpu):
    torch, b = gpu
    q, s = b.gspc_quantize_rows_f8(torch.zeros(0, 40, device="cuda"))
    assert q.shape == (0, 128) and s.shape == (0, 4)
    assert b.gspc_dequantize_rows_f8((q, s), 40).shape == (0, 40)
    x = torch.randn(3, 5, 200, device="cuda")
    rows, columns = b.gspc_quantize_rows_f8(x, which=b.F8_BOTH)
    for one, two in ((rows, b.gspc_quantize_rows_f8(x)), (columns, b.gspc_quantize_rows_f8(x, which=b.F8_COLUMNS)),
                     (columns, b.gspc_quantize_rows_f8(x.view(15, 200).t().contiguous()))):
        assert torch.equal(one[0].view(torch.uint8), two[0].view(torch.uint8)) and torch.equal(one[1], two[1])


def test_a_byte_of_255_is_no_number(gpu):
    """Rows that another program wrote: a power of two that is none makes its block no number, in what is read and in products of either type."""
    torch, b = gpu
    a, w = b.gspc_quantize_rows_f8(torch.randn(40, 256, device="cuda")), b.gspc_quantize_rows_f8(torch.randn(24, 256, device="cuda"))
    a[1][7, 1] = 255
    back = b.gspc_dequantize_rows_f8(a, 256)
    assert bool(back[7, 128:].isnan().all()) and int(back.isnan().sum()) == 128
    for dtype in (b.GSPC_F32, b.GSPC_BF16):
        out = b.gspc_matmul_f8(a, w, dtype=dtype)
        assert bool(out[7].isnan().all()) and int(out.isnan().sum()) == 24


# ---- products ------------------------------------------------------------------------------------------
def product_inputs(torch, b, rng, M, K, N, spread=1.0):
    a = rng.standard_normal((M, K)) * np.exp2(np.rint(spread * rng.standard_normal((M, 1)) * 4))
    w = rng.standard_normal((N, K)) * np.exp2(np.rint(spread * rng.standard_normal((N, 1)) * 4))
    for v in (a, w):                                            # blocks of a row with powers of their own
        for k in range(0, K, 128):
            v[:, k:k + 128] *= 2.0 ** rng.integers(-3, 4)
    return [b.gspc_quantize_rows_f8(dev(torch, v.astype(np.float32))) for v in (a, w)]


def check_product(out, a, w, bias, K, bf16):
    (qa, ca), (qw, cw) = a, w
    x, y = f8_read(qa, ca), f8_read(qw, cw)
    want, size = x @ y.T, np.abs(x) @ np.abs(y).T
    if bias is not None:
        want = want + bias
    tol = (K * 2.0 ** -23 + (2.0 ** -10 if bf16 else 0)) * size + (B if bf16 else U) * np.abs(want) * (1 + 2.0 ** -7) + 1e-38
    err = np.abs(out - want)
    assert (err <= tol).all(), np.max(err / tol)
    return want, size


SHAPES = [(1, 1, 1), (1, 16, 1), (2, 7, 3), (1, 4096, 512), (3, 129, 17), (16, 128, 16), (17, 200, 33), (33, 640, 31), (65, 512, 130), (64, 1024, 128),
          (5, 5000, 70), (130, 1280, 1001), (197, 333, 250), (257, 512, 257), (513, 384, 300), (100, 128, 5000), (2000, 100, 48), (300, 4000, 300),
          (129, 8192, 129), (1024, 2048, 1100), (64, 20000, 64)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("to", ["float32", "bfloat16"])
def test_product(gpu, shape, to):
    torch, b = gpu
    M, K, N = shape
    rng = np.random.default_rng(M + 3 * K + 7 * N)
    a, w = product_inputs(torch, b, rng, M, K, N)
    bias = rng.standard_normal(N).astype(np.float32) if (M + N) % 2 else None
    kind = b.GSPC_F32 if to == "float32" else b.GSPC_BF16
    out = b.gspc_matmul_f8(a, w, None if bias is None else dev(torch, bias), dtype=kind, cols=K)
    check_product(host(out), values(torch, a), values(torch, w), bias, K, to == "bfloat16")
    wide = torch.full((M + 2, N + 6), 5.0, dtype=out.dtype, device="cuda")
    b.gspc_matmul_f8(a, w, None if bias is None else dev(torch, bias), out=wide[1:-1, 3:-3])
    assert torch.equal(wide[1:-1, 3:-3], out)
    wide[1:-1, 3:-3] = 5.0
    assert bool((wide == 5.0).all())


# every tile: from few tokens to many, sums cut into stretches, outputs past the caches
TILES = [(8, 4096, 4096, "product_f8_small<1,1>"), (3, 4200, 20001, "product_f8_small<1,1>"), (9, 4200, 20001, "product_f8_tile<64,128>"),
         (200, 1024, 1024, "product_f8_small<2,2>"), (1000, 2000, 3000, "product_f8_tile<128,128>"), (512, 4096, 4096, "product_f8_tile<64,128>"),
         (2048, 512, 4096, "product_f8_tile<128,128>"), (3000, 640, 4100, "product_f8_tile<256,256>")]


@pytest.mark.parametrize("M,K,N,kernel", TILES)
def test_every_tile(gpu, M, K, N, kernel):
    torch, b = gpu
    rng = np.random.default_rng(M)
    a, w = product_inputs(torch, b, rng, M, K, N, 0.3)
    out = b.gspc_matmul_f8(a, w)
    assert b.gspc_last_kernel() == kernel
    check_product(host(out), values(torch, a), values(torch, w), None, K, True)
    assert torch.equal(b.gspc_matmul_f8(a, w), out)             # the same bits again
    check_product(host(b.gspc_matmul_f8(a, w, dtype=b.GSPC_F32)), values(torch, a), values(torch, w), None, K, False)


@pytest.mark.parametrize("M,K,N", [(96, 16384, 160), (256, 50176, 128), (64, 20000, 300), (1, 65536, 40), (300, 6400, 520), (200, 9000, 333)])
@pytest.mark.parametrize("to", ["float32", "bfloat16"])
def test_long_sums_of_few_outputs(gpu, M, K, N, to):
    """A weight's gradient sums over all tokens: stretches of them, joined.  The workspace is as large as said, and what it held does not matter."""
    torch, b = gpu
    rng = np.random.default_rng(M + N)
    a, w = product_inputs(torch, b, rng, M, K, N, 0.1)
    need = b.gspc_matmul_f8_workspace_bytes(M, N, K)
    assert need > 0 and need % 4 == 0
    whole = torch.full((need // 4 + 64,), float("nan"), device="cuda")
    whole[need // 4:] = 7.0
    bias = rng.standard_normal(N).astype(np.float32)
    kind = b.GSPC_F32 if to == "float32" else b.GSPC_BF16
    out = b.gspc_matmul_f8(a, w, dev(torch, bias), dtype=kind, workspace=whole[:need // 4])
    assert bool((whole[need // 4:] == 7.0).all())
    check_product(host(out), values(torch, a), values(torch, w), bias, K, to == "bfloat16")
    assert torch.equal(b.gspc_matmul_f8(a, w, dev(torch, bias), dtype=kind), out)
    with pytest.raises(b.GspcError, match="SPACE"):
        b.gspc_matmul_f8(a, w, dev(torch, bias), dtype=b.GSPC_F32, workspace=whole[:need // 4 - 1])


@pytest.mark.parametrize("M,K,N", [(1, 300, 40), (130, 640, 260), (600, 4096, 512)])
def test_powers_of_two_at_the_ends_of_their_range(gpu, M, K, N):
    """Blocks scaled by powers from 2^-127 to 2^100, whose products are ordinary numbers."""
    torch, b = gpu
    rng = np.random.default_rng(K)
    e = rng.integers(-100, 100, (K + 127) // 128).repeat(128)[:K]
    e[:128] = -118
    a = (rng.standard_normal((M, K)) * np.exp2(e)).astype(np.float32)
    w = (rng.standard_normal((N, K)) * np.exp2(-e)).astype(np.float32)
    a, w = (b.gspc_quantize_rows_f8(dev(torch, v)) for v in (a, w))
    for kind in (b.GSPC_F32, b.GSPC_BF16):
        check_product(host(b.gspc_matmul_f8(a, w, dtype=kind)), values(torch, a), values(torch, w), None, K, kind == b.GSPC_BF16)


@pytest.mark.parametrize("M,N", [(2, 126), (300, 520), (2048, 4096)])
@pytest.mark.parametrize("power", [-127, -126, -125, -124, -118, -60, 0, 118])
def test_every_code_at_the_ends_of_the_range(gpu, M, N, power):
    """All positive codes times powers of two, one a filter: to fp32 exact in blocks of 2^-124 and more, and below within half of 2^-133."""
    torch, b = gpu
    codes = torch.zeros(128)
    codes[:126] = torch.arange(1, 127).to(torch.uint8).view(torch.float8_e4m3fn).float()
    x = (codes.double() * 2.0 ** power).float().cuda().repeat(M, 1)
    other = 100 if power < 0 else -100
    w = torch.zeros(N, 128)
    w[torch.arange(126), torch.arange(126)] = 2.0 ** other
    a = b.gspc_quantize_rows_f8(x)
    assert bool((a[1][:, 0] == power + 127).all()) and torch.equal(a[0][0].float().cpu(), codes)
    want = codes[:126].double() * 2.0 ** (power + other)
    out = b.gspc_matmul_f8(a, b.gspc_quantize_rows_f8(w.cuda()), dtype=b.GSPC_F32)
    assert bool((out == out[:1]).all()) and not bool(out[:, 126:].any())
    off = (out[0, :126].cpu().double() - want).abs().max().item()
    assert off <= (2.0 ** (-134 + other) if power < -124 else 0)
    assert torch.equal(b.gspc_matmul_f8(a, b.gspc_quantize_rows_f8(w.cuda()))[0, :126].cpu(), want.bfloat16())


def test_values_past_the_largest_number(gpu):
    """What 3.4 x 10^38 is rounded to is 2^128: a number to bf16 outputs, and an infinity to fp32 outputs and to what reads it."""
    torch, b = gpu
    a = b.gspc_quantize_rows_f8(torch.full((2, 128), 3.4e38, device="cuda"))
    w = b.gspc_quantize_rows_f8(torch.full((40, 128), 2.0 ** -100, device="cuda"))
    assert bool((b.gspc_matmul_f8(a, w) == 2.0 ** 35).all()) and bool((b.gspc_matmul_f8(a, w, dtype=b.GSPC_F32) == float("inf")).all())
    for dtype in (b.GSPC_F32, b.GSPC_BF16):
        assert bool((b.gspc_dequantize_rows_f8(a, 128, dtype=dtype) == float("inf")).all())


@pytest.mark.parametrize("M,K,N", [(3, 200, 40), (300, 640, 520), (2048, 256, 4096)])
def test_what_is_not_finite_stays_in_its_outputs(gpu, M, K, N):
    torch, b = gpu
    x, y = torch.randn(M, K, device="cuda"), torch.randn(N, K, device="cuda")
    x[1, 3], y[17, K - 1] = float("nan"), float("inf")
    for kind in (b.GSPC_F32, b.GSPC_BF16):
        out = b.gspc_matmul_f8(b.gspc_quantize_rows_f8(x), b.gspc_quantize_rows_f8(y), dtype=kind)
        bad = out.isnan()
        assert bool(bad[1].all()) and bool(bad[:, 17].all()) and int(bad.sum()) == N + M - 1


def test_gradients_of_a_product_are_products(gpu):
    """y = x w^T: dx from dy's rows and w's columns form, dw from dy's and x's columns forms, against the gradients of the rows' values; and those of
    whole numbers, which e4m3 holds, against torch's own."""
    torch, b = gpu
    for whole in (False, True):
        M, K, N = 700, 200, 130
        g = torch.Generator(device="cuda").manual_seed(1)
        make = lambda *s: torch.randint(-8, 9, s, device="cuda", generator=g).float() if whole else torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        x, w, dy = make(M, K), make(N, K), make(M, N)
        (xr, xc), (wr, wc), (dr, dc) = (b.gspc_quantize_rows_f8(t, which=b.F8_BOTH) for t in (x, w, dy))
        y, dx, dw = (b.gspc_matmul_f8(*p, dtype=b.GSPC_F32) for p in ((xr, wr), (dr, wc), (dc, xc)))
        for out, (p, q), length in ((y, (xr, wr), K), (dx, (dr, wc), N), (dw, (dc, xc), M)):
            check_product(host(out), values(torch, p), values(torch, q), None, length, False)
        if whole:
            x, w = x.cpu().requires_grad_(), w.cpu().requires_grad_()
            (x @ w.t()).backward(dy.cpu())
            assert torch.equal(dx.cpu(), x.grad) and torch.equal(dw.cpu(), w.grad)     # (exact: sums below 2^24)


def test_f8_side_stream_and_replayed_graph(gpu):
    torch, b = gpu
    x, w = torch.randn(300, 4000, device="cuda").bfloat16(), torch.randn(300, 4000, device="cuda")

    def work():
        rows, columns = b.gspc_quantize_rows_f8(x, which=b.F8_BOTH)
        return b.gspc_matmul_f8(rows, b.gspc_quantize_rows_f8(w)), columns[0].view(torch.uint8), columns[1]

    want = [t.clone() for t in work()]
    with on_side_stream(torch, b) as s:
        got = work()
        s.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = work()
        for k in range(3):
            x.copy_(torch.randn_like(x))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            again = work()
            s.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(held, again)), k


def test_rows_and_products_past_32_bits(gpu):
    """Tensors of more than 2^32 elements: the first and the last rows get, bit by bit, what they get by themselves."""
    torch, b = gpu
    C, some = 512, 4096
    rows = (1 << 32) // C + some
    small = torch.randn(some, C, device="cuda").bfloat16()
    x = small.repeat(rows // some, 1)
    assert x.numel() > 1 << 32
    q, want = b.gspc_quantize_rows_f8(x), b.gspc_quantize_rows_f8(small)
    for t, v in zip(q, want):
        t, v = t.view(torch.uint8), v.view(torch.uint8)
        assert torch.equal(t[:some], v) and torch.equal(t[-some:], v)
    b.gspc_dequantize_rows_f8(q, C, out=x)
    back = b.gspc_dequantize_rows_f8(want, C, dtype=b.GSPC_BF16)
    assert torch.equal(x[:some], back) and torch.equal(x[-some:], back)
    w = b.gspc_quantize_rows_f8(torch.randn(C, C, device="cuda"))
    b.gspc_matmul_f8(q, w, out=x)
    y = b.gspc_matmul_f8(want, w)
    assert torch.equal(x[:some], y) and torch.equal(x[-some:], y)
    del q
    x = small.repeat(rows // some, 1)
    _, columns = b.gspc_quantize_rows_f8(x, which=b.F8_BOTH)
    pitch = b.gspc_f8_pitch(some)
    want = b.gspc_quantize_rows_f8(small, which=b.F8_COLUMNS)
    assert torch.equal(columns[0][:, :pitch].view(torch.uint8), want[0].view(torch.uint8))
    assert torch.equal(columns[0][:, -pitch:].view(torch.uint8), want[0].view(torch.uint8))
    assert torch.equal(columns[1][:, :32], want[1]) and torch.equal(columns[1][:, rows // 128 - 32:rows // 128], want[1])
