"""A residual block's operators: argument errors are found on the host before any GPU work (these calls return before the first HIP call),
and the sizes that the library reports."""
import ctypes

import pytest

from paper_2006_09791_amd import binding as b

P = ctypes.c_void_p(256 * 1024)                 # never dereferenced: validation fails first, or there is no work
Q = ctypes.c_void_p(512 * 1024)
ODD1, ODD2, ODD4, ODD8 = (ctypes.c_void_p(256 * 1024 + k) for k in (1, 2, 4, 8))
NULL, DIM, GROUPS, DTYPE, SPACE, ARG, MISMATCH = -1, -2, -3, -4, -6, -8, -5


def refused(call, good, bad):
    for at, value, code in bad:
        args = list(good)
        args[at] = value
        assert call(*args) == code, (at, value)


def test_pitches():
    lib = b.load()
    for cols, pitch, scales in ((1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (513, 640, 8), (4096, 4096, 32)):
        assert lib.gspc_f8_pitch(cols) == b.gspc_f8_pitch(cols) == pitch
        assert lib.gspc_f8_scale_pitch(cols) == b.gspc_f8_scale_pitch(cols) == scales
    for cols in (0, -3, 0x7fffffff, 0x7ffffc01):
        assert lib.gspc_f8_pitch(cols) == lib.gspc_f8_scale_pitch(cols) == 0 and "columns" in b.gspc_last_error()
        for call in (b.gspc_f8_pitch, b.gspc_f8_scale_pitch):
            with pytest.raises(b.GspcError):
                call(cols)
    assert lib.gspc_f8_pitch(0x7ffffc00) == 0x7ffffc00


def test_rows_refusals():
    lib = b.load()
    # x, dtype, ldx, rows, cols, q, scale, qt, scale_t
    refused(lib.gspc_quantize_rows_f8, [P, 0, 40, 3, 40, P, P, P, P],
            [(0, None, NULL), (0, ODD2, ARG), (1, 2, DTYPE), (1, 3, DTYPE), (2, 39, DIM), (3, -1, DIM), (3, 1 << 31, DIM), (3, 0x7ffffc01, DIM), (4, 0, DIM),
             (4, 0x7ffffc01, DIM), (5, ODD8, ARG), (6, None, NULL), (6, ODD2, ARG), (7, ODD8, ARG), (8, None, NULL), (8, ODD1, ARG)])
    assert lib.gspc_quantize_rows_f8(P, 0, 40, 3, 40, None, None, None, None) == NULL
    assert lib.gspc_quantize_rows_f8(P, 0, 0x7ffffc00, 0x7ffffc00, 0x7ffffc00, P, P, P, P) == DIM
    assert lib.gspc_quantize_rows_f8(None, 0, 40, 0, 40, None, None, None, None) == 0
    refused(lib.gspc_dequantize_rows_f8, [P, P, 3, 40, P, 0, 40],
            [(0, None, NULL), (0, ODD8, ARG), (1, None, NULL), (1, ODD2, ARG), (2, -1, DIM), (3, 0, DIM), (4, None, NULL), (4, ODD2, ARG), (5, 3, DTYPE),
             (6, 39, DIM)])
    assert lib.gspc_dequantize_rows_f8(None, None, 0, 40, None, 0, 40) == 0


def test_product_refusals():
    lib = b.load()
    # a, a_scale, w, w_scale, bias, M, N, K, out, dtype, ldo, workspace, bytes
    refused(lib.gspc_matmul_f8, [P, P, P, P, None, 5, 7, 33, P, 0, 7, None, 0],
            [(0, None, NULL), (0, ODD8, ARG), (1, None, NULL), (1, ODD2, ARG), (2, None, NULL), (2, ODD8, ARG), (3, None, NULL), (3, ODD1, ARG),
             (4, ODD2, ARG), (5, -1, DIM), (5, 1 << 31, DIM), (6, 0, DIM), (7, 0, DIM), (7, (1 << 22) + 1, DIM), (8, None, NULL), (8, ODD2, ARG),
             (9, 3, DTYPE), (10, 6, DIM), (11, ODD8, ARG)])
    assert lib.gspc_matmul_f8(None, None, None, None, None, 0, 7, 33, None, 0, 7, None, 0) == 0
    need = lib.gspc_matmul_f8_workspace_bytes(256, 128, 50176)
    assert need >= 2 * 256 * 128 * 4
    good = [P, P, P, P, None, 256, 128, 50176, P, 0, 128, P, need]
    refused(lib.gspc_matmul_f8, good, [(11, None, NULL), (11, ODD8, ARG), (12, need - 1, SPACE), (12, 0, SPACE)])
    assert lib.gspc_matmul_f8_workspace_bytes(0, 128, 50176) == lib.gspc_matmul_f8_workspace_bytes(4096, 4096, 4096) == 0
    for bad in ((-1, 7, 33), (5, 0, 33), (5, 7, 0), (5, 7, (1 << 22) + 1), (1 << 31, 7, 33)):
        b.load().gspc_last_error()
        assert lib.gspc_matmul_f8_workspace_bytes(*bad) == 0 and "M=" in b.gspc_last_error()


def test_dropout_refusals():
    lib = b.load()
    # x, dtype, ldx, rows, cols, drop, seed, offset, step, y, ldy
    refused(lib.gspc_dropout, [P, 0, 40, 3, 40, 0.5, 1, 2, P, Q, 40],
            [(0, None, NULL), (0, ODD2, ARG), (1, 2, DTYPE), (2, 39, DIM), (3, -1, DIM), (4, 0, DIM), (5, -0.1, ARG), (5, 1.1, ARG), (5, float("nan"), ARG),
             (8, ODD4, ARG), (9, None, NULL), (9, ODD2, ARG), (10, 39, DIM)])
    assert lib.gspc_dropout(P, 0, 48, 3, 40, 0.5, 1, 2, None, P, 40) == ARG        # in place, rows another distance apart
    assert lib.gspc_dropout(None, 0, 40, 0, 40, 0.5, 1, 2, None, None, 40) == 0


def description(**change):
    r = b.GspcResidual(12, 3, 40, b.NORM_LAYER, b.NORM_RMS, b.ACT_SILU, P, P, P, P, P, 1.0, 1e-5, 0.5, 1, 2, P)
    for k, v in change.items():
        setattr(r, k, v)
    return r


BAD = [(dict(rows=-1), DIM), (dict(rows=1 << 31), DIM), (dict(rows=13), GROUPS), (dict(gates=0), GROUPS), (dict(gates=-3), GROUPS), (dict(cols=0), DIM),
       (dict(cols=8193), DIM), (dict(post=3), ARG), (dict(pre=-1), ARG), (dict(act=3), ARG), (dict(post=0), ARG), (dict(pre=0), ARG),
       (dict(pre=0, pre_gamma=None, pre_beta=None), ARG), (dict(post_gamma=ODD2), ARG), (dict(post_beta=ODD1), ARG), (dict(pre_gamma=ODD2), ARG),
       (dict(pre_beta=ODD2), ARG), (dict(gate=ODD2), ARG), (dict(drop=1.5), ARG), (dict(drop=float("nan")), ARG), (dict(step=ODD4), ARG)]


def test_residual_refusals():
    lib = b.load()
    # r, x, dtype, ldx, h, dtype, ldh, xo, ldxo, z, dtype, ldz, z_scale, stats
    good = [description(), P, 0, 40, P, 1, 40, Q, 40, Q, 1, 40, None, P]
    refused(lib.gspc_residual_norm, good, [(0, None, NULL)] + [(0, description(**c), code) for c, code in BAD] +
            [(0, description(eps=e), ARG) for e in (0.0, -1.0, float("inf"), float("nan"))] +
            [(1, None, NULL), (1, ODD2, ARG), (2, 2, DTYPE), (3, 39, DIM), (4, None, ARG), (4, ODD1, ARG), (5, 3, DTYPE), (6, 39, DIM), (7, ODD2, ARG),
             (8, 39, DIM), (9, ODD1, ARG), (10, 2, DTYPE), (11, 39, DIM), (13, ODD8, ARG)])
    args = list(good)
    args[10] = b.GSPC_F8                        # 8-bit float rows without scales, and misaligned ones
    assert lib.gspc_residual_norm(*args) == NULL
    args[9] = ODD8
    assert lib.gspc_residual_norm(*args) == ARG
    args = list(good)
    args[7] = args[9] = None                    # nothing to write
    assert lib.gspc_residual_norm(*args) == NULL
    args = list(good)
    args[7], args[8] = P, 48                    # in place, rows another distance apart
    assert lib.gspc_residual_norm(*args) == ARG
    plain = dict(pre=0, pre_gamma=None, pre_beta=None, act=0)
    assert lib.gspc_residual_norm(description(**plain), *good[1:]) == ARG                  # z of no norm
    assert lib.gspc_residual_norm(description(rows=0), None, 0, 40, None, 1, 40, None, 40, None, 1, 40, None, None) == 0


def test_residual_gradient_refusals():
    lib = b.load()
    need = lib.gspc_residual_norm_backward_workspace_bytes(12, 40, 3)
    assert need > 0
    # r, dz, dtype, ld, dxo, ld, xo, dtype, ld, h, dtype, ld, stats, dx, ld, dh, ld, dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta, workspace, bytes
    good = [description(), P, 1, 40, P, 40, P, 0, 40, P, 1, 40, P, Q, 40, Q, 40, P, P, P, P, P, P, need]
    refused(lib.gspc_residual_norm_backward, good, [(0, None, NULL)] + [(0, description(**c), code) for c, code in BAD] +
            [(1, ODD1, ARG), (2, 2, DTYPE), (3, 39, DIM), (4, ODD2, ARG), (5, 39, DIM), (6, None, NULL), (6, ODD2, ARG), (7, 3, DTYPE), (8, 39, DIM),
             (9, None, ARG), (9, ODD1, ARG), (10, 2, DTYPE), (11, 39, DIM), (12, None, NULL), (12, ODD8, ARG), (13, None, NULL), (13, ODD2, ARG), (14, 39, DIM),
             (15, None, NULL), (15, ODD1, ARG), (16, 39, DIM), (17, ODD2, ARG), (18, ODD2, ARG), (19, ODD1, ARG), (20, ODD2, ARG), (21, ODD2, ARG),
             (22, None, NULL), (22, ODD8, ARG), (23, need - 1, SPACE)])
    args = list(good)
    args[1] = args[4] = None                    # neither gradient
    assert lib.gspc_residual_norm_backward(*args) == NULL
    for at, ld in ((4, 14), (9, 16)):           # in place, rows another distance apart
        args = list(good)
        args[{4: 13, 9: 15}[at]], args[ld] = args[at], 48
        assert lib.gspc_residual_norm_backward(*args) == ARG
    for change in (dict(pre=0, pre_gamma=None, pre_beta=None, act=0), dict(post=0, post_gamma=None, post_beta=None), dict(gate=None)):
        assert lib.gspc_residual_norm_backward(description(**change), *good[1:]) == ARG     # gradients of what is not there
    for bad in ((-1, 40, 3), (12, 0, 3), (12, 8193, 3), (12, 40, 0), (12, 40, 5), (1 << 31, 40, 1)):
        assert lib.gspc_residual_norm_backward_workspace_bytes(*bad) == 0 and "gates" in b.gspc_last_error()
    assert lib.gspc_residual_norm_backward_workspace_bytes(0, 40, 3) == 0


class TestBinding:
    """What the Python calls refuse by themselves."""
    torch = pytest.importorskip("torch")

    class Fake(torch.Tensor):
        """A host tensor that says it is on the GPU: what is refused for its shape or type never gets to be read."""
        is_cuda = True

    def fake(self, *shape, dtype=torch.float32):
        return self.torch.zeros(shape).to(dtype).as_subclass(self.Fake)

    def rows8(self, rows, cols):
        return (self.fake(rows, b.gspc_f8_pitch(cols), dtype=self.torch.float8_e4m3fn), self.fake(rows, b.gspc_f8_scale_pitch(cols), dtype=self.torch.uint8))

    def test_host_tensors(self):
        t = self.torch
        x, pair = t.zeros(6, 40), (t.zeros(6, 128).to(t.float8_e4m3fn), t.zeros(6, 4, dtype=t.uint8))
        for call in (lambda: b.gspc_quantize_rows_f8(x), lambda: b.gspc_quantize_rows_f8(x, out=pair), lambda: b.gspc_dequantize_rows_f8(pair, 40),
                     lambda: b.gspc_matmul_f8(pair, pair), lambda: b.gspc_dropout(x, 0.5, 0), lambda: b.gspc_dropout(x, 0.5, 0, out=x),
                     lambda: b.gspc_residual_norm(x, x, out=x, xo=x, pre=1), lambda: b.gspc_residual_norm(x, pre=1),
                     lambda: b.gspc_residual_norm_backward(None, x, x, None, t.zeros(6, 4), dx=x)):
            with pytest.raises(b.GspcError, match="GPU"):
                call()

    def test_shapes_and_types(self):
        t, f = self.torch, self.fake
        x, r8 = f(6, 40), self.rows8(6, 40)
        half = f(6, 40, dtype=t.float16)
        cases = [
            (lambda: b.gspc_quantize_rows_f8(f(6, 0)), "no columns"), (lambda: b.gspc_quantize_rows_f8(f(0, 40), which=b.F8_COLUMNS), "no rows"),
            (lambda: b.gspc_quantize_rows_f8(x, which=4), "forms"), (lambda: b.gspc_quantize_rows_f8(x, out=r8, which=b.F8_COLUMNS), "forms"),
            (lambda: b.gspc_quantize_rows_f8(x, out=self.rows8(7, 40)), "768"), (lambda: b.gspc_quantize_rows_f8(half, out=r8), "neither"),
            (lambda: b.gspc_quantize_rows_f8(x, out_t=r8), "out_t"),
            (lambda: b.gspc_dequantize_rows_f8(r8, 40, out=f(6, 41)), "expected 6 rows of 40"),
            (lambda: b.gspc_matmul_f8(r8, self.rows8(5, 129)), "filters of 256"), (lambda: b.gspc_matmul_f8(r8, self.rows8(5, 40), cols=129), "pitch"),
            (lambda: b.gspc_matmul_f8(r8, self.rows8(5, 40), out=f(6, 4)), "expected 6 rows of 5"),
            (lambda: b.gspc_matmul_f8(r8, self.rows8(5, 40), bias=f(6), out=f(6, 5)), "bias"),
            (lambda: b.gspc_matmul_f8((f(6, 40, dtype=t.float8_e4m3fn), r8[1]), (f(5, 40, dtype=t.float8_e4m3fn), r8[1])), "pitch"),
            (lambda: b.gspc_dropout(f(6, 0), 0.5, 0), "no columns"), (lambda: b.gspc_dropout(x, 0.5, 0, out=f(40, 6)), "shape"),
            (lambda: b.gspc_dropout(x, 0.5, 0, out=f(6, 40, dtype=t.bfloat16)), "bfloat16"), (lambda: b.gspc_dropout(x, 0.5, -1, out=f(6, 40)), "64 bits"),
            (lambda: b.gspc_dropout(x, 0.5, 0, 1 << 64, out=f(6, 40)), "64 bits"), (lambda: b.gspc_dropout(x, 0.5, 0.5, out=f(6, 40)), "64 bits"),
            (lambda: b.gspc_dropout(x, 0.5, 0, step=f(1), out=f(6, 40)), "step"), (lambda: b.gspc_dropout(x, 1.5, 0, out=f(6, 40)), "probability"),
            (lambda: b.gspc_residual_norm(f(6, 0)), "no channels"), (lambda: b.gspc_residual_norm(x, f(6, 41), xo=f(6, 40)), "h has shape"),
            (lambda: b.gspc_residual_norm(x, f(5, 40), xo=f(6, 40)), "h has shape"), (lambda: b.gspc_residual_norm(x, f(6, 40), xo=f(6, 41)), "xo has shape"),
            (lambda: b.gspc_residual_norm(x, f(6, 40), xo=f(6, 40, dtype=t.bfloat16)), "xo is"),
            (lambda: b.gspc_residual_norm(x, f(6, 40), gate=f(3, 41), xo=f(6, 40)), "gate has shape"),
            (lambda: b.gspc_residual_norm(x, f(6, 40), gate=f(4, 40), xo=f(6, 40)), "divisible"),
            (lambda: b.gspc_residual_norm(x, f(6, 40), gate=f(3, 40, dtype=t.bfloat16), xo=f(6, 40)), "gate"),
            (lambda: b.gspc_residual_norm(x, pre=1, pre_gamma=f(41), out=f(6, 40)), "pre_gamma"), (lambda: b.gspc_residual_norm(x, pre=1, out=f(6, 41)), "out has"),
            (lambda: b.gspc_residual_norm(x, pre=1, out=f(6, 40), stats=f(6, 3)), "stats"),
            (lambda: b.gspc_residual_norm(x, pre=1, out=self.rows8(6, 129)), "out"),
            (lambda: b.gspc_residual_norm(f(6, 8200), pre=1, out=f(6, 8200)), "channels"),
            (lambda: b.gspc_residual_norm(x, out=f(6, 40)), "no norm"),
            (lambda: b.gspc_residual_norm_backward(None, None, None, None, f(6, 4)), "neither"),
            (lambda: b.gspc_residual_norm_backward(None, f(5, 40), x, None, f(6, 4), dx=f(6, 40)), "dxo has shape"),
            (lambda: b.gspc_residual_norm_backward(None, f(6, 40, dtype=t.bfloat16), x, None, f(6, 4), dx=f(6, 40)), "dxo is"),
            (lambda: b.gspc_residual_norm_backward(None, x, x, None, f(6, 3), dx=f(6, 40), workspace=f(9000)), "stats"),
            (lambda: b.gspc_residual_norm_backward(None, x, x, x, f(6, 4), dx=f(6, 40), dh=f(6, 40, dtype=t.bfloat16)), "dh is"),
            (lambda: b.gspc_residual_norm_backward(None, x, x, x, f(6, 4), gate=f(3, 40), dx=f(6, 40), dh=f(6, 40), dgate=f(2, 40), workspace=f(9000)), "dgate")]
        for call, match in cases:
            with pytest.raises(b.GspcError, match=match):
                call()
