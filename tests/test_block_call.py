"""The C form of the residual block's calls: what arrives at the library, argument by argument, and what is left to the general route."""
import ctypes
import types

import pytest

from paper_2006_09791_amd import binding as b

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2006_09791_amd._gspc_call")
I, P, L, D, U, Z, R = (ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_double, ctypes.c_uint64, ctypes.c_size_t, ctypes.POINTER(b.GspcResidual))
PROTOTYPES = [  # quantize, dequantize, matmul, dropout, residual_norm, residual_norm_backward
    [P, I, L, L, I, P, P, P, P], [P, P, L, I, P, I, L], [P, P, P, P, P, L, I, I, P, I, L, P, Z], [P, I, L, L, I, D, U, U, P, P, L],
    [R, P, I, L, P, I, L, P, L, P, I, L, P, P], [R, P, I, L, P, L, P, I, L, P, I, L, P, P, L, P, L, P, P, P, P, P, P, Z]]
LIBRARY = ["gspc_quantize_rows_f8", "gspc_dequantize_rows_f8", "gspc_matmul_f8", "gspc_dropout", "gspc_residual_norm", "gspc_residual_norm_backward",
           "gspc_matmul_f8_workspace_bytes", "gspc_residual_norm_backward_workspace_bytes"]
TYPES = torch.float8_e4m3fn, torch.uint8, torch.int64
BF, F8, U8, I64 = torch.bfloat16, *TYPES


def fake(at, shape, dtype=torch.float32, cuda=True, contiguous=True):
    return types.SimpleNamespace(is_cuda=cuda, dtype=dtype, shape=torch.Size(shape), is_contiguous=lambda: contiguous, data_ptr=lambda: at)


def fields(r):
    return tuple(getattr(r, name) for name, _ in b.GspcResidual._fields_)


@pytest.fixture
def call():
    """(the module, the list of calls that arrived as (number, arguments), descriptions as tuples)."""
    lib = b.load()
    from paper_2006_09791_amd import _gspc_call
    seen, keep = [], []

    def recorder(k):
        def take(*a):
            seen.append((k, (fields(a[0].contents), *a[1:]) if k > 3 else a))
            return -100 - k
        return ctypes.CFUNCTYPE(I, *PROTOTYPES[k])(take)
    for k in range(6):
        keep.append(recorder(k))
    sizes = ctypes.CFUNCTYPE(Z, L, I, I)(lambda *a: sum(a)), ctypes.CFUNCTYPE(Z, L, I, L)(lambda *a: sum(a))
    bind = lambda fs: _gspc_call.bind_block(*[ctypes.cast(f, P).value for f in fs], *TYPES)  # noqa: E731
    bind(keep + list(sizes))
    try:
        yield _gspc_call, seen
    finally:
        bind([getattr(lib, n) for n in LIBRARY])


def rows8(at, rows, cols):
    return fake(at, (rows, (cols + 127) // 128 * 128), F8), fake(at + 1, (rows, (cols + 511) // 512 * 4), U8)


def test_arguments_arrive(call):
    c, seen = call
    n = None
    assert c.quantize_f8(fake(16, (4, 7, 200), BF), rows8(64, 28, 200), rows8(96, 200, 28)) == -100
    assert c.quantize_f8(fake(16, (28, 200)), None, rows8(96, 200, 28)) == c.quantize_f8(fake(16, (28, 200)), rows8(64, 28, 200), None) == -100
    assert c.dequantize_f8(rows8(64, 28, 200), 200, fake(16, (4, 7, 200), BF)) == -101
    assert c.matmul_f8(rows8(64, 6, 600), rows8(128, 9, 600), fake(512, (9,)), fake(1024, (2, 3, 9), BF), 600, fake(320, (50,)), None) == -102
    made, out = [], fake(1024, (6, 9))
    make = lambda n, like: made.append((n, like)) or fake(640, (n,), U8)  # noqa: E731
    assert c.matmul_f8(rows8(64, 6, 600), rows8(128, 9, 600), None, out, None, None, make) == -102 and made == [(6 + 9 + 640, out)]
    assert c.dropout(fake(16, (2, 3, 9), BF), 0.25, (1 << 64) - 1, 7, fake(40, (1,), I64), fake(32, (2, 3, 9), BF)) == -103
    x, h, g, v = fake(16, (2, 5, 24), BF), fake(32, (2, 5, 24)), fake(48, (5, 24)), [fake(100 + k, (24,)) for k in range(4)]
    assert c.residual_norm(x, h, g, 2, v[0], v[1], 1, v[2], v[3], 2, 0.5, 0.25, 0.125, 8, 9, fake(40, (), I64), fake(80, (2, 5, 24), BF), fake(96, (2, 5, 24)),
                           fake(112, (10, 4))) == -104
    assert c.residual_norm(x, None, None, 0, None, None, 1, None, None, 0, 1.0, 0.25, 0.0, 0, 0, None, None, rows8(64, 10, 24), None) == -104
    assert c.residual_norm_backward(fake(17, (2, 5, 24)), fake(18, (2, 5, 24), BF), x, h, fake(112, (10, 4)), g, 2, v[0], v[1], 1, v[2], v[3], 2, 0.5, 0.125, 8, 9,
                                    None, fake(19, (2, 5, 24), BF), fake(20, (2, 5, 24)), fake(21, (5, 24)), *[fake(30 + k, (24,)) for k in range(4)],
                                    fake(320, (50,)), None) == -105
    dx = fake(19, (2, 5, 24), BF)
    assert c.residual_norm_backward(None, x, None, None, fake(112, (10, 4)), None, 0, None, None, 0, None, None, 0, 1.0, 0.0, 0, 0, None, dx,
                                    None, None, None, None, None, None, None, make) == -105 and made[1:] == [(10 + 24 + 1, dx)]
    eps = ctypes.c_float(0.25).value
    assert seen == [
        (0, (16, 1, 200, 28, 200, 64, 65, 96, 97)), (0, (16, 0, 200, 28, 200, n, n, 96, 97)), (0, (16, 0, 200, 28, 200, 64, 65, n, n)),
        (1, (64, 65, 28, 200, 16, 1, 200)),
        (2, (64, 65, 128, 129, 512, 6, 9, 640, 1024, 1, 9, 320, 200)), (2, (64, 65, 128, 129, n, 6, 9, 640, 1024, 0, 9, 640, 655)),
        (3, (16, 1, 9, 6, 9, 0.25, (1 << 64) - 1, 7, 40, 32, 9)),
        (4, ((10, 5, 24, 2, 1, 2, 100, 101, 102, 103, 48, 0.5, eps, 0.125, 8, 9, 40), 16, 1, 24, 32, 0, 24, 80, 24, 96, 0, 24, n, 112)),
        (4, ((10, 1, 24, 0, 1, 0, n, n, n, n, n, 1.0, eps, 0.0, 0, 0, n), 16, 1, 24, n, 0, 24, n, 24, 64, 3, 24, 65, n)),
        (5, ((10, 5, 24, 2, 1, 2, 100, 101, 102, 103, 48, 0.5, 1.0, 0.125, 8, 9, n), 17, 0, 24, 18, 24, 16, 1, 24, 32, 0, 24, 112, 19, 24, 20, 24, 21,
             30, 31, 32, 33, 320, 200)),
        (5, ((10, 1, 24, 0, 0, 0, n, n, n, n, n, 1.0, 1.0, 0.0, 0, 0, n), n, 0, 24, 16, 24, n, 1, 24, n, 0, 24, 112, 19, 24, n, 24, n, n, n, n, n, 640, 35))]


def left(c, call, good, bad):
    for at, value in bad:
        args = list(good)
        args[at] = value
        assert call(*args) is NotImplemented, (at, value)
    assert call(*good[:-1]) is NotImplemented


def test_what_is_left_to_the_general_route(call):
    c, seen = call
    x, q, qt = fake(16, (28, 200)), rows8(64, 28, 200), rows8(96, 200, 28)
    other = [fake(16, (28, 200), cuda=False), fake(16, (28, 200), contiguous=False), fake(16, (28, 200), torch.float64), fake(16, (28, 200), F8), None, 7]
    left(c, c.quantize_f8, [x, q, qt], [(0, o) for o in other] + [(0, fake(16, (0, 200))), (0, fake(16, (28, 0))), (1, list(q)), (1, qt), (1, q[:1]), (2, q),
                                                                 (1, (fake(1, (28, 256), U8), q[1])), (1, (q[0], fake(1, (28, 8), U8)))])
    left(c, c.dequantize_f8, [q, 200, x], [(0, qt), (0, None), (0, list(q)), (1, 201), (1, 200.0), (1, 0)] + [(2, o) for o in other])
    a, w, out = rows8(64, 6, 600), rows8(128, 9, 600), fake(1024, (6, 9))
    left(c, c.matmul_f8, [a, w, None, out, 600, fake(320, (50,)), None],
         [(0, rows8(64, 7, 600)), (0, rows8(64, 6, 700)), (0, list(a)), (0, (fake(64, (3840,), F8), a[1])), (0, (fake(64, (6, 600), F8), a[1])),
          (0, (a[0], fake(65, (6, 4), U8))), (1, rows8(128, 8, 600)), (2, fake(512, (8,))), (2, fake(512, (9,), BF)), (3, None), (3, fake(1024, (6, 8))),
          (3, fake(1024, (6, 9), F8)), (4, 641), (4, 0), (4, 600.0), (5, 7), (5, fake(320, (9,), contiguous=False))])
    left(c, c.dropout, [x, 0.5, 1, 2, None, x], [(0, o) for o in other] + [(0, fake(16, (28, 0))), (1, 1), (1, None), (2, -1), (2, 1 << 64), (2, 1.0), (3, -1), (3, None),
                                                                          (4, 7), (4, fake(40, (2,), I64)), (4, fake(40, (1,))), (5, None), (5, fake(32, (28, 201))),
                                                                          (5, fake(32, (28, 200), BF)), (5, fake(32, (200, 28)))])
    x, v, st = fake(16, (10, 24)), fake(100, (24,)), fake(112, (10, 4))
    left(c, c.residual_norm, [x, x, v, 2, v, v, 1, v, v, 2, 0.5, 0.25, 0.125, 8, 9, None, x, x, st],
         [(0, None), (0, fake(16, (10, 0))), (0, fake(16, (10, 8200))), (1, fake(32, (10, 25))), (1, fake(32, (5, 2, 24))), (2, fake(48, (25,))),
          (2, fake(48, (24,), BF)), (3, "2"), (4, fake(1, (23,))), (5, 7), (6, 1 << 40), (7, fake(1, (24,), BF)), (8, x), (9, None), (10, 1), (11, 1), (12, 0),
          (13, -1), (14, 0.0), (15, x), (16, fake(80, (10, 24), BF)), (16, fake(80, (24, 10))), (17, None), (17, fake(96, (10, 23))), (17, rows8(64, 9, 24)),
          (17, list(rows8(64, 10, 24))), (18, fake(112, (10, 3)))])
    left(c, c.residual_norm_backward, [x, x, x, x, st, v, 2, v, v, 1, v, v, 2, 0.5, 0.125, 8, 9, None, x, x, v, v, v, v, v, fake(320, (50,)), None],
         [(0, fake(16, (10, 23))), (1, fake(16, (10, 24), BF)), (2, fake(16, (10, 24), BF)), (3, fake(16, (9, 24))), (4, None), (4, fake(112, (10, 3))),
          (5, fake(48, (25,))), (13, 1), (14, None), (15, 1.0), (17, st), (18, None), (18, fake(16, (10, 8200))), (19, fake(16, (10, 24), BF)),
          (19, None), (20, None), (22, None), (20, fake(1, (48,))), (21, fake(1, (23,))), (24, 7), (25, 7)])
    assert not seen
    with pytest.raises(ZeroDivisionError):      # a workspace that cannot be made: its error, and no call
        c.matmul_f8(a, w, None, out, 600, None, lambda n, like: 1 // 0)
    assert c.matmul_f8(a, w, None, out, 600, None, lambda n, like: 7) is NotImplemented and not seen
