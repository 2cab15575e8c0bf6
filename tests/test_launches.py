"""How the channels-last operators are cut into launches: no launch has 2^32 threads or more, which the HIP runtime refuses, and the
launches of a call together reach every image once."""
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
