"""Channels-last operators: argument errors are found on the host before any GPU work (these calls return before the first
HIP call), and the sizes that the library reports."""
import ctypes

import pytest

from paper_2006_09791_amd import binding as b

P = ctypes.c_void_p(256 * 1024)                 # never dereferenced: validation fails first, or there is no work
ODD2, ODD4, ODD8 = (ctypes.c_void_p(256 * 1024 + k) for k in (1, 2, 8))
NULL, DIM, GROUPS, DTYPE, SPACE, ARG, MISMATCH = -1, -2, -3, -4, -6, -8, -5


def test_pitch():
    lib = b.load()
    for cols, pitch in ((1, 16), (15, 16), (16, 16), (17, 32), (333, 336), (4096, 4096)):
        assert lib.gspc_rows8_pitch(cols) == b.gspc_rows8_pitch(cols) == pitch
    assert lib.gspc_rows8_pitch(0) == lib.gspc_rows8_pitch(-3) == lib.gspc_rows8_pitch(0x7fffffff) == 0
    assert "columns" in b.gspc_last_error()
    with pytest.raises(b.GspcError):
        b.gspc_rows8_pitch(0)


@pytest.mark.parametrize("name", ["gspc_pack_channels_last", "gspc_unpack_channels_last"])
def test_layout_refusals(name):
    call = getattr(b.load(), name)
    good = [P, 0, 2, 8, 9, P, 1]
    for at, value, code in ((2, -1, DIM), (3, 0, DIM), (4, -5, DIM), (1, 2, DTYPE), (6, 7, DTYPE), (0, None, NULL), (5, None, NULL),
                            (0, ODD4, ARG), (5, ODD2, ARG)):
        args = list(good)
        args[at] = value
        assert call(*args) == code, (at, value)
    assert call(None, 0, 0, 8, 9, None, 1) == call(None, 0, 2, 8, 0, None, 1) == 0
    assert call(P, 0, 2, 0x7fffffff, 0x7fffffff, P, 1) == DIM


def test_rows_refusals():
    lib = b.load()
    good = [P, 0, 40, 3, 40, P, P]              # x, dtype, ldx, rows, cols, q, scale
    for at, value, code in ((1, 2, DTYPE), (2, 39, DIM), (3, -1, DIM), (3, 1 << 31, DIM), (4, 0, DIM), (4, 0x7fffffff, DIM), (0, None, NULL),
                            (5, None, NULL), (6, None, NULL), (0, ODD4, ARG), (5, ODD8, ARG), (6, ODD4, ARG)):
        args = list(good)
        args[at] = value
        assert lib.gspc_quantize_rows(*args) == code, (at, value)
        x, dtype, ldx, rows, cols, q, scale = args
        assert lib.gspc_dequantize_rows(q, scale, rows, cols, x, dtype, ldx) == code, (at, value)
    assert lib.gspc_quantize_rows(None, 0, 40, 0, 40, None, None) == 0
    assert lib.gspc_dequantize_rows(None, None, 0, 40, None, 0, 40) == 0


def test_norm_refusals():
    lib = b.load()
    need = lib.gspc_group_norm_workspace_bytes(1, 70000, 8, 1, 0, 0)
    assert need > 0
    # x, dtype, ldx, gamma, beta, N, P, C, groups, eps, act, y, dtype, ldy, y_scale, stats, saved, saved_scale, workspace, bytes
    good = [P, 0, 32, P, P, 1, 70000, 8, 1, 1e-5, 0, P, 0, 32, None, None, None, None, P, need]
    bad = [(0, None, NULL), (0, ODD4, ARG), (1, 2, DTYPE), (2, 7, DIM), (3, ODD4, ARG), (5, -1, DIM), (6, -1, DIM), (7, 0, DIM),
           (8, 5, GROUPS), (8, 0, GROUPS), (9, 0.0, ARG), (9, float("nan"), ARG), (9, float("inf"), ARG), (9, -1.0, ARG), (10, 3, ARG),
           (11, None, NULL), (11, ODD4, ARG), (12, 9, DTYPE), (13, 7, DIM), (15, ODD4, ARG), (16, P, NULL), (16, ODD8, ARG),
           (18, None, NULL), (18, ODD8, ARG), (19, need - 1, SPACE)]
    for at, value, code in bad:
        args = list(good)
        args[at] = value
        assert lib.gspc_group_norm(*args) == code, (at, value)
    args = list(good)
    args[12] = b.GSPC_I8                        # 8-bit rows without scales, and misaligned ones
    assert lib.gspc_group_norm(*args) == NULL
    args[11] = ODD8
    assert lib.gspc_group_norm(*args) == ARG
    for at in (5, 6):                           # nothing to do
        args = [None, 0, 32, None, None, 2, 9, 32, 4, 1e-5, 0, None, 0, 32, None, None, None, None, None, 0]
        args[at] = 0
        assert lib.gspc_group_norm(*args) == 0


def test_norm_backward_refusals():
    lib = b.load()
    need = lib.gspc_group_norm_backward_workspace_bytes(2, 9, 32, 4, 0, 0)
    assert need > 0
    # dy, dtype, lddy, x, dtype, ldx, x_scale, stats, gamma, beta, N, P, C, groups, act, dx, lddx, dgamma, dbeta, workspace, bytes
    good = [P, 0, 32, P, 0, 32, None, P, P, P, 2, 9, 32, 4, 0, P, 32, P, P, P, need]
    bad = [(0, None, NULL), (0, ODD4, ARG), (1, 2, DTYPE), (2, 8, DIM), (3, None, NULL), (4, 5, DTYPE), (4, 2, NULL), (5, 31, DIM),
           (7, None, NULL), (7, ODD4, ARG), (8, ODD4, ARG), (10, -1, DIM), (12, -8, DIM), (13, 3, GROUPS), (14, -1, ARG),
           (15, None, NULL), (16, 31, DIM), (17, ODD4, ARG), (18, ODD2, ARG), (19, None, NULL), (19, ODD8, ARG), (20, need - 1, SPACE)]
    for at, value, code in bad:
        args = list(good)
        args[at] = value
        assert lib.gspc_group_norm_backward(*args) == code, (at, value)


def test_workspace_sizes():
    lib = b.load()
    forward, backward = lib.gspc_group_norm_workspace_bytes, lib.gspc_group_norm_backward_workspace_bytes
    assert forward(0, 9, 32, 4, 0, 0) == backward(2, 0, 32, 4, 0, 0) == 0
    assert forward(2, 9, 32, 5, 0, 0) == 0 and "divisible" in b.gspc_last_error()
    assert backward(65536, 65536, 8, 1, 0, 0) == 0 and "tokens" in b.gspc_last_error()
    assert forward(2, 9, 32, 4, 2, 0) == 0 and "dtype" in b.gspc_last_error()
    assert backward(2, 9, 32, 4, 2, 0) == backward(2, 9, 32, 4, 0, 3) == 0
    # images that a block holds: nothing but the statistics behind 8-bit rows, and sums of several images
    assert forward(2, 9, 32, 4, 0, 0) == 0 and forward(2, 9, 32, 4, 0, 1) == 2 * 4 * 8
    assert backward(1, 9, 32, 4, 0, 0) == 0 and backward(2, 9, 32, 4, 1, 2) == 2 * 2 * 32 * 4
    # images that it does not hold: parts of the sums as well
    assert forward(1, 70000, 8, 1, 0, 0) > 8 and backward(1, 70000, 8, 1, 0, 0) > 2 * 8 * 4


def test_product_refusals():
    lib = b.load()
    good = [P, P, P, P, None, 5, 7, 33, P, 0, 7]    # a, a_scale, w, w_scale, bias, M, N, K, out, dtype, ldo
    for at, value, code in ((0, None, NULL), (0, ODD8, ARG), (1, None, NULL), (1, ODD4, ARG), (2, None, NULL), (2, ODD8, ARG), (3, None, NULL),
                            (4, ODD4, ARG), (5, -1, DIM), (5, 1 << 31, DIM), (6, 0, DIM), (7, 0, DIM), (7, 133145, DIM), (8, None, NULL),
                            (8, ODD4, ARG), (9, 2, DTYPE), (10, 6, DIM)):
        args = list(good)
        args[at] = value
        assert lib.gspc_matmul_i8(*args) == code, (at, value)
    assert lib.gspc_matmul_i8(None, None, None, None, None, 0, 7, 33, None, 0, 7) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 32)
    for call in (lambda: b.gspc_quantize_rows(x), lambda: b.gspc_pack_channels_last(x),
                 lambda: b.gspc_group_norm(x, None, None, 4, out=x),
                 lambda: b.gspc_matmul_i8((torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2)),
                                          (torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3)), out=torch.zeros(2, 3))):
        with pytest.raises(b.GspcError, match="GPU"):
            call()
    with pytest.raises(b.GspcError, match="filters of 32"):
        b.gspc_matmul_i8((torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2)), (torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3)))
