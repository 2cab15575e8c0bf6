"""How the channels-last operators are cut into launches: no launch has 2^32 threads or more, which the HIP runtime refuses, and the
launches of a call together reach every image once."""
import re
import struct

import pytest

import fake_runtime

BASE = 1 << 40                  # addresses that nothing reads
OUT = 1 << 44


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    return fake_runtime.build(tmp_path_factory.mktemp("runtime"))


def pointer(raw):
    return struct.unpack("<Q", raw)[0]


LAYOUT = {"transpose_kernel": [(0, 8), (1, 8), (9, 4)], "transpose_thin_kernel": [(0, 8), (1, 8)]}


@pytest.mark.parametrize("call,C,P", [(c, C, P) for c in ("gspc_pack_channels_last", "gspc_unpack_channels_last")
                                      for C, P in ((8, 8), (3, 2), (3, 9), (9, 3), (64, 1), (70, 130))])
@pytest.mark.parametrize("N", [1, 300, 17_000_000])
def test_layout_launches_reach_every_image(runtime, call, C, P, N):
    (rc, found), = fake_runtime.launches(runtime, [(call, [BASE, 0, N, C, P, OUT, 1])], LAYOUT)
    assert rc == 0
    thin = (C < 8) != (P < 8)
    tiles = (max(C, P) + 1023) // 1024 if thin else ((C + 63) // 64) * ((P + 63) // 64)
    at = 0
    for kernel, blocks, threads, args in found:
        assert kernel == ("transpose_thin_kernel" if thin else "transpose_kernel") and blocks * threads < 1 << 32
        assert pointer(args[0]) == BASE + 4 * at * C * P and pointer(args[1]) == OUT + 2 * at * C * P
        assert blocks % tiles == 0
        at += blocks // tiles
    assert at == N and (N > 300 or len(found) == 1)


def test_layout_launches_of_one_large_plane(runtime):
    """A plane of more tiles than a launch may have blocks: its tiles are numbered on."""
    N, C, P = 2, 8, 0x7fffffff
    (rc, found), = fake_runtime.launches(runtime, [("gspc_pack_channels_last", [BASE, 1, N, C, P, OUT, 1])], LAYOUT)
    assert rc == 0
    tiles, at = (P + 63) // 64, 0
    for _, blocks, threads, args in found:
        assert blocks * threads < 1 << 32
        image, first = divmod(at, tiles)
        assert pointer(args[0]) == BASE + 2 * image * C * P and pointer(args[1]) == OUT + 2 * image * C * P
        assert struct.unpack("<I", args[2])[0] == first and first + blocks <= tiles
        at += blocks
    assert at == N * tiles


# What the norm's kernels are given: NormShape (N first), and the pointers that go from image to image.
NORM = {"norm_stats_kernel": [(0, 4), (2, 8), (4, 8)], "norm_join_kernel": [(0, 4), (2, 8), (4, 8)],
        "norm_apply_kernel": [(0, 4), (2, 8), (6, 8), (9, 8)], "norm_rows_kernel": [(0, 4), (5, 8), (7, 8), (10, 8), (12, 8), (13, 8), (14, 8)],
        "norm_held_kernel": [(0, 4)],
        "norm_grad_sums_kernel": [(0, 4), (2, 8), (4, 8), (6, 8), (7, 8), (10, 8)], "norm_grad_join_kernel": [(0, 4), (3, 8), (5, 8), (6, 8)],
        "norm_grad_apply_kernel": [(0, 4), (2, 8), (4, 8), (6, 8), (7, 8), (10, 8), (11, 8), (14, 4), (15, 4)], "norm_grad_params_kernel": [(0, 4), (1, 4)]}
X, Y, YS, ST, SV, SS, DX, DG, DB, WS = (BASE + (k << 41) for k in range(10))       # (tensors are below 2^41 bytes)


def number(raw):
    return int.from_bytes(raw, "little")


def consecutive(found, kernel, N, per_image):
    """The launches of `kernel` take the N images in turn, and its pointers go `per_image` bytes (first address, step) with them."""
    at, some = 0, [f for f in found if f[0] == kernel]
    for _, blocks, threads, args in some:
        assert blocks * threads < 1 << 32
        for raw, (base, step) in zip(args[1:], per_image):
            assert number(raw) == (base + at * step if base else 0), kernel
        at += number(args[0])
    assert at == N, kernel
    return some


# N, P, C, groups: blocks of one row for each image; 448 threads for images of seven channels; 256 threads and two slabs
MANY_IMAGES = [(17_000_000, 1, 16, 1), (9_600_000, 64, 7, 1), (5_000_000, 1, 2056, 1)]


@pytest.mark.parametrize("N,P,C,groups", MANY_IMAGES)
@pytest.mark.parametrize("kind", ["dense", "rows8", "saved"])
def test_norm_launches_reach_every_image(runtime, N, P, C, groups, kind):
    pitch, rows = (C + 15) // 16 * 16, kind == "rows8"
    need = fake_runtime.b.gspc_group_norm_workspace_bytes(N, P, C, groups, 1, kind != "dense")
    saved = (SV, SS) if kind == "saved" else (None, None)
    (rc, found), = fake_runtime.launches(runtime, [("gspc_group_norm", [X, 1, C, None, None, N, P, C, groups, 1e-5, 2, Y, 2 if rows else 1, C,
                                                                        YS if rows else None, ST, *saved, WS, need])], NORM)
    assert rc == 0
    x, st = (X, 2 * P * C), (ST, 8 * groups)
    slabs = (C + 2047) // 2048
    first = WS                                                  # of the parts: the statistics are the caller's
    consecutive(found, "norm_stats_kernel", N, [x, (first, 8 * (groups + slabs - 1))])
    consecutive(found, "norm_join_kernel", N, [(first, 8 * (groups + slabs - 1)), st])
    if kind == "dense":
        consecutive(found, "norm_apply_kernel", N, [x, st, (Y, 2 * P * C)])
    else:
        y = (Y, P * pitch) if rows else (Y, 2 * P * C)
        some = consecutive(found, "norm_rows_kernel", N, [x, st, y, (YS if rows else 0, 4 * P), (saved[0] or 0, P * pitch), (saved[1] or 0, 4 * P)])
        assert all(blocks == number(args[0]) for _, blocks, _, args in some)


@pytest.mark.parametrize("N,P,C,groups", MANY_IMAGES + [(1, 1, 1 << 28, 1 << 20), (2, 3, (1 << 30) + 8, 1)])
@pytest.mark.parametrize("rows8", [False, True])
def test_gradient_launches_reach_every_image(runtime, N, P, C, groups, rows8):
    pitch = (C + 15) // 16 * 16
    need = fake_runtime.b.gspc_group_norm_backward_workspace_bytes(N, P, C, groups, 1, 2 if rows8 else 1)
    (rc, found), = fake_runtime.launches(runtime, [("gspc_group_norm_backward", [Y, 1, C, X, 2 if rows8 else 1, C, YS if rows8 else None, ST, None, None,
                                                                                 N, P, C, groups, 2, DX, C, DG, DB, WS, need])], NORM)
    assert rc == 0
    for _, blocks, threads, _ in found:
        assert blocks * threads < 1 << 32
    if any(k == "norm_grad_held_kernel" for k, *_ in found):
        return
    x, dy, scale, st = (X, P * pitch if rows8 else 2 * P * C), (Y, 2 * P * C), (YS if rows8 else 0, 4 * P), (ST, 8 * groups)
    sums, ab, parts = (WS, 8 * C), (WS + 8 * C * N, 8 * groups), (WS + 8 * C * N + 8 * groups * N, 8 * C)
    assert found[-1][0] == "norm_grad_apply_kernel" and parts[0] + parts[1] * N <= WS + need
    consecutive(found, "norm_grad_sums_kernel", N, [dy, x, scale, st, parts])
    consecutive(found, "norm_grad_join_kernel", N, [parts, sums, ab])
    some = consecutive(found, "norm_grad_apply_kernel", N, [dy, x, scale, st, ab, (DX, 2 * P * C)])
    with_params = [args for *_, args in some if number(args[7])]
    assert len(with_params) == 1 and number(with_params[0][8]) == N


def test_gradients_of_many_parameters_without_tokens(runtime):
    (rc, found), = fake_runtime.launches(runtime, [("gspc_group_norm_backward", [None, 1, 1 << 30, None, 1, 1 << 30, None, None, None, None,
                                                                                 0, 3, 1 << 30, 1, 2, None, 1 << 30, DG, DB, None, 0])], NORM)
    assert rc == 0 and len(found) == 1 and found[0][1] * found[0][2] < 1 << 32


PRODUCT = {k: [(-1, 0), (0, 88)] for k in ("product8_small_kernel", "product8_tile_kernel")}


def product_tile(raw):
    """(tokens, filters) of a block, from the kernel's name."""
    n = [int(v) for v in re.findall(r"Li(\d+)E", raw.decode())]
    return (32 * n[0] * n[2], 32 * n[1] * n[3]) if b"tile_kernel" in raw else (16 * n[1], 16 * n[0])


@pytest.mark.parametrize("M,N", [(1, 50257), (16, 128256), (17, 50257), (64, 33000), (64, 1 << 20), (65, 33000), (100, 50257), (128, 128256), (50000, 1),
                                 (50000, 10), (200000, 64), (50000, 100), (1 << 20, 128), (129, 50257), (50000, 129), (8192, 8192), (12544, 1024)])
@pytest.mark.parametrize("K", [128, 4096])
def test_large_tiles_are_at_least_half_full(runtime, M, N, K):
    """A tile of 128 tokens and more, or of 256 filters, is taken where the product fills more than half of it."""
    (rc, found), = fake_runtime.launches(runtime, [("gspc_matmul_i8", [X, SV, Y, YS, None, M, N, K, DX, 1, N])], PRODUCT)
    assert rc == 0
    for _, _, _, (name, _) in found:
        tokens, filters = product_tile(name)
        assert tokens < 128 or 2 * M > tokens, (tokens, filters)
        assert filters < 256 or 2 * N > filters, (tokens, filters)


@pytest.mark.parametrize("M,N", [(0x7fffffff, 100), (0x7fffffff, 130), (0x7fffffff, 200), (1 << 30, 1), (1, 0x7ffffff0), (16, 140_000_000), (64, 0x7ffffff0),
                                 (100, 0x7ffffff0), (3, 5), (8192, 8192)])
@pytest.mark.parametrize("bias", [None, SS])
def test_product_launches_cover_the_output(runtime, M, N, bias):
    K, ld = 16, N + 3
    (rc, found), = fake_runtime.launches(runtime, [("gspc_matmul_i8", [X, SV, Y, YS, bias, M, N, K, DX, 1, ld])], PRODUCT)
    assert rc == 0
    seen = set()
    for _, blocks, threads, (name, raw) in found:
        assert blocks * threads < 1 << 32
        a, w, sa, sw, sb, out, m, ldo, n, pitch, mtiles, ntiles, _ = struct.unpack("<8Q2i2Ii", raw[:84])
        m0, n0 = (a - X) // pitch, (w - Y) // pitch
        assert (a, w, sa, sw, out) == (X + m0 * pitch, Y + n0 * pitch, SV + 4 * m0, YS + 4 * n0, DX + 2 * (m0 * ld + n0))
        assert sb == (bias + 4 * n0 if bias else 0) and ldo == ld and pitch == K
        tokens, filters = product_tile(name)
        assert (mtiles, ntiles) == (-(-m // tokens), -(-n // filters)) and blocks == mtiles * ntiles
        assert m0 + m <= M and n0 + n <= N and m0 % tokens == 0 and n0 % filters == 0
        seen.add((m0, n0, m * n))
    assert len(seen) == len(found) and sum(s for *_, s in seen) == M * N


PAST = {"transpose_kernel": [(8, 4)], "transpose_thin_kernel": [(7, 4)], "norm_apply_kernel": [(11, 4)], "norm_held_kernel": [(10, 4)],
        "norm_rows_kernel": [(15, 4)], "norm_grad_held_kernel": [(15, 4)], "norm_grad_apply_kernel": [(13, 4)], "dequantize_rows_kernel": [(7, 4)]}


def goes_past(runtime, name, args):
    """Whether the kernel that writes the call's output is told to write past the caches."""
    (rc, found), = fake_runtime.launches(runtime, [(name, args)], {**PAST, **PRODUCT})
    assert rc == 0
    if name == "gspc_matmul_i8":
        return bool(struct.unpack("<i", found[-1][3][1][80:84])[0])
    return bool(number([args for k, _, _, args in found if k in PAST][-1][0]))


@pytest.mark.parametrize("N,P,C,groups", [(64, 3136, 96, 8), (256, 784, 64, 8), (128, 3136, 24, 4)])
def test_norms_write_whole_pieces_past_the_caches(runtime, N, P, C, groups):
    """bf16 side by side, or in rows of whole pieces of 64 bytes; never fp32, whose vectors are two stores with a gap."""
    def forward(ld, kind=1, saved=None, at=0):
        need = fake_runtime.b.gspc_group_norm_workspace_bytes(N, P, C, groups, kind, saved is not None)
        return goes_past(runtime, "gspc_group_norm", [X, kind, C, None, None, N, P, C, groups, 1e-5, 2, Y + at, kind, ld, None, ST, saved, SS, WS, need])

    def backward(ld, kind=1, at=0):
        need = fake_runtime.b.gspc_group_norm_backward_workspace_bytes(N, P, C, groups, kind, kind)
        return goes_past(runtime, "gspc_group_norm_backward", [Y, kind, C, X, kind, C, None, ST, None, None, N, P, C, groups, 2, DX + at, ld, DG, DB, WS, need])

    whole = C % 32 == 0
    for call in (forward, backward, lambda *a, **k: forward(*a, saved=SV, **k)):
        assert call(C) and call(C, at=2) and call(2 * C) == call(C + 32) == whole
        assert not (call(C + 2) or call(C + 16) or call(2 * C, at=32) or call(C, kind=0) or call(2 * C, kind=0))


def test_gradients_of_wide_rows_go_past_the_caches(runtime):
    need = fake_runtime.b.gspc_group_norm_backward_workspace_bytes(64, 3136, 256, 32, 1, 1)
    assert goes_past(runtime, "gspc_group_norm_backward", [Y, 1, 256, X, 1, 256, None, ST, None, None, 64, 3136, 256, 32, 2, DX, 258, DG, DB, WS, need])


@pytest.mark.parametrize("M,N,K", [(100000, 128, 64), (16384, 1024, 256), (8192, 8192, 4096), (100000, 256, 64)])
def test_products_write_whole_pieces_past_the_caches(runtime, M, N, K):
    call = lambda N, ld, kind, at=0: goes_past(runtime, "gspc_matmul_i8", [X, SV, Y, YS, None, M, N, K, DX + at, kind, ld])  # noqa: E731
    for kind, line in ((1, 32), (0, 16)):
        assert call(N, N, kind) and call(N, N + line, kind) and call(N - line, N, kind)
        assert not (call(N, N + 1, kind) or call(N, N + 8, kind) or call(N - 1, N - 1, kind) or call(N - 4, N, kind) or call(N, N, kind, 16))


@pytest.mark.parametrize("name,C,P,past", [("gspc_pack_channels_last", 128, 784, True), ("gspc_pack_channels_last", 100, 1073, False),
                                           ("gspc_pack_channels_last", 32, 3136, False), ("gspc_unpack_channels_last", 128, 784, False),
                                           ("gspc_unpack_channels_last", 128, 3136, True), ("gspc_pack_channels_last", 6, 12545, True),
                                           ("gspc_unpack_channels_last", 6, 12544, True), ("gspc_unpack_channels_last", 6, 12545, False)])
def test_layout_passes_write_whole_pieces_past_the_caches(runtime, name, C, P, past):
    assert goes_past(runtime, name, [X, 0, 256, C, P, Y, 1]) == past
    assert not goes_past(runtime, name, [X, 1, 256, C, P, Y, 0])         # fp32
    assert not goes_past(runtime, name, [X, 0, 1, C, P, Y, 1])           # small


def test_norm_given_statistics_needs_no_workspace_for_them(runtime):
    """In two passes: the parts' bytes alone, from the workspace's start on."""
    N, P, C, groups = 3, 70000, 8, 2
    need, own = fake_runtime.b.gspc_group_norm_workspace_bytes(N, P, C, groups, 0), 8 * N * groups
    call = lambda stats, given: ("gspc_group_norm", [X, 0, C, None, None, N, P, C, groups, 1e-5, 0, Y, 0, C, None, stats, None, None, WS, given])  # noqa: E731
    results = fake_runtime.launches(runtime, [call(None, need - 1), call(ST, need - own - 1), call(None, need), call(ST, need - own)], NORM)
    assert [rc for rc, _ in results] == [-6, -6, 0, 0]
    for (_, found), first in zip(results[2:], (WS + own, WS)):
        assert number([args for k, _, _, args in found if k == "norm_stats_kernel"][0][2]) == first
        assert number([args for k, _, _, args in found if k == "norm_apply_kernel"][0][3]) == Y


GRIDS = {"norm_stats_kernel": [(0, 28), (1, 40)], "norm_apply_kernel": [(0, 28), (1, 40)], "norm_grad_sums_kernel": [(0, 28), (1, 40)],
         "norm_grad_apply_kernel": [(0, 28), (1, 40)], "norm_rows_kernel": [(2, 4), (3, 4)]}


@pytest.mark.parametrize("P", [0x7fffffff, 0x7fffffff - 300, 0x7fffffff - (1 << 18), 0x7fffffff - (1 << 23), 1 << 30])
@pytest.mark.parametrize("C", [1, 8, 24, 2056])
@pytest.mark.parametrize("N", [1, 2])
def test_long_images_are_cut_into_all_of_their_rows(runtime, N, P, C):
    """Up to 2^31 - 1 tokens: rows of a block times blocks reach the last one, and no block begins past it."""
    if N * P > 0x7fffffff:
        P //= N
    b = fake_runtime.b
    need = [b.gspc_group_norm_workspace_bytes(N, P, C, 1, 1, rows8) for rows8 in (0, 1)] + [b.gspc_group_norm_backward_workspace_bytes(N, P, C, 1, 1, 1)]
    norm = lambda kind, need: ("gspc_group_norm", [X, 1, C, None, None, N, P, C, 1, 1e-5, 2, Y, kind, C, YS, None, None, None, WS, need])  # noqa: E731
    back = ("gspc_group_norm_backward", [Y, 1, C, X, 1, C, None, ST, None, None, N, P, C, 1, 2, DX, C, DG, DB, WS, need[2]])
    for rc, found in fake_runtime.launches(runtime, [norm(1, need[0]), norm(2, need[1]), back], GRIDS):
        assert rc == 0 and not any("held" in k for k, *_ in found)
        for kernel, blocks, threads, args in found:
            if kernel == "norm_rows_kernel":
                chunks, rows = map(number, args)
                assert blocks == N * chunks
            elif args:
                slabs, (chunks, rows) = struct.unpack("<i", args[1][4:8])[0], struct.unpack("<2i", args[1][20:28])
                assert blocks >= N * chunks * slabs
            else:
                continue
            assert (chunks - 1) * rows < P <= chunks * rows, kernel
