"""The C form of the channels-last operators' calls: what arrives at the library, argument by argument, and what is left to the
general route."""
import ctypes
import types

import pytest

from paper_2006_09791_amd import binding as b

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2006_09791_amd._gspc_call")
I, P, L, F, Z = ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
PROTOTYPES = [  # pack, unpack, quantize, dequantize, norm, norm_backward, matmul
    [P, I, I, I, I, P, I], [P, I, I, I, I, P, I], [P, I, L, L, I, P, P], [P, P, L, I, P, I, L],
    [P, I, L, P, P, I, I, I, I, F, I, P, I, L, P, P, P, P, P, Z],
    [P, I, L, P, I, L, P, P, P, P, I, I, I, I, I, P, L, P, P, P, Z],
    [P, P, P, P, P, L, I, I, P, I, L]]
LIBRARY = ["gspc_pack_channels_last", "gspc_unpack_channels_last", "gspc_quantize_rows", "gspc_dequantize_rows", "gspc_group_norm",
           "gspc_group_norm_backward", "gspc_matmul_i8"]


def fake(at, shape, dtype=torch.float32, cuda=True, contiguous=True):
    return types.SimpleNamespace(is_cuda=cuda, dtype=dtype, shape=torch.Size(shape), is_contiguous=lambda: contiguous, data_ptr=lambda: at)


@pytest.fixture
def call():
    """(the module, the list of calls that arrived as (number, arguments))."""
    lib = b.load()
    from paper_2006_09791_amd import _gspc_call
    seen, keep = [], []

    def recorder(k):
        return ctypes.CFUNCTYPE(I, *PROTOTYPES[k])(lambda *a: seen.append((k, a)) or -100 - k)
    for k in range(7):
        keep.append(recorder(k))
    bind = lambda fs: _gspc_call.bind_tokens(*[ctypes.cast(f, P).value for f in fs], torch.float32, torch.bfloat16, torch.int8)  # noqa: E731
    bind(keep)
    try:
        yield _gspc_call, seen
    finally:
        bind([getattr(lib, n) for n in LIBRARY])


def rows8(at, rows, cols):
    return fake(at, (rows, (cols + 15) // 16 * 16), torch.int8), fake(at + 1, (rows,))


def test_arguments_arrive(call):
    c, seen = call
    bf = torch.bfloat16
    assert c.pack(fake(16, (2, 3, 5)), fake(32, (2, 5, 3), bf)) == -100
    assert c.unpack(fake(16, (2, 5, 3), bf), fake(32, (2, 3, 5))) == -101
    assert c.quantize(fake(16, (4, 7, 33), bf), rows8(64, 28, 33)) == -102
    assert c.dequantize(rows8(64, 28, 33), 33, fake(16, (28, 33))) == -103
    x, g, h, stats = fake(16, (2, 5, 24), bf), fake(48, (24,)), fake(52, (24,)), fake(80, (2, 3, 2))
    assert c.norm(x, g, h, 3, 0.5, 2, fake(96, (2, 5, 24)), stats, rows8(160, 10, 24), fake(320, (100,), torch.int8)) == -104
    assert c.norm(x, None, None, 3, 0.5, 1, rows8(160, 10, 24), None, None, None) == -104
    assert c.norm_backward(fake(16, (2, 5, 24)), rows8(160, 10, 24), stats, g, h, 3, 2, fake(96, (2, 5, 24)), fake(112, (24,)), fake(116, (24,)), None) == -105
    assert c.norm_backward(fake(16, (2, 5, 24)), x, stats, None, None, 3, 2, fake(96, (2, 5, 24)), fake(112, (24,)), fake(116, (24,)), fake(320, (50,))) == -105
    assert c.matmul(rows8(64, 6, 40), rows8(128, 9, 40), fake(512, (9,)), fake(1024, (2, 3, 9), bf)) == -106
    n = None
    assert seen == [
        (0, (16, 0, 2, 3, 5, 32, 1)), (1, (16, 1, 2, 3, 5, 32, 0)), (2, (16, 1, 33, 28, 33, 64, 65)), (3, (64, 65, 28, 33, 16, 0, 33)),
        (4, (16, 1, 24, 48, 52, 2, 5, 24, 3, 0.5, 2, 96, 0, 24, n, 80, 160, 161, 320, 100)),
        (4, (16, 1, 24, n, n, 2, 5, 24, 3, 0.5, 1, 160, 2, 24, 161, n, n, n, n, 0)),
        (5, (16, 0, 24, 160, 2, 24, 161, 80, 48, 52, 2, 5, 24, 3, 2, 96, 24, 112, 116, n, 0)),
        (5, (16, 0, 24, 16, 1, 24, n, 80, n, n, 2, 5, 24, 3, 2, 96, 24, 112, 116, 320, 200)),
        (6, (64, 65, 128, 129, 512, 6, 9, 48, 1024, 1, 9))]


def test_what_is_left_to_the_general_route(call):
    c, seen = call
    bf, i8 = torch.bfloat16, torch.int8
    x, y = fake(16, (2, 3, 5)), fake(32, (2, 5, 3), bf)
    for bad in (fake(16, (2, 3, 5), cuda=False), fake(16, (2, 3, 5), contiguous=False), fake(16, (2, 3, 5), torch.float64), fake(16, (2, 3, 5), i8),
                fake(16, (2, 3, 4)), fake(16, (6, 5)), fake(16, (0, 3, 5)), None, 7, types.SimpleNamespace(is_cuda=True)):
        assert c.pack(bad, y) is NotImplemented
    assert c.pack(x) is c.pack(x, None) is c.unpack(x, fake(32, (2, 5, 3), i8)) is NotImplemented
    q = rows8(64, 28, 33)
    for bad in (None, list(q), q[:1], (q[0], fake(1, (27,))), (fake(1, (28, 33), i8), q[1]), (fake(1, (28, 48)), q[1]), (q[0], fake(1, (28,), bf))):
        assert c.quantize(fake(16, (28, 33)), bad) is c.dequantize(bad, 33, fake(16, (28, 33))) is NotImplemented
    assert c.dequantize(q, 34, fake(16, (28, 33))) is c.dequantize(q, 33.0, fake(16, (28, 33))) is NotImplemented
    x, g, stats, out = fake(16, (2, 5, 24)), fake(48, (24,)), fake(80, (2, 3, 2)), fake(96, (2, 5, 24))
    good = [x, g, g, 3, 1e-5, 0, out, stats, None, None]
    for at, bad in ((0, fake(16, (10, 24))), (0, fake(16, (2, 0, 24))), (1, fake(48, (23,))), (2, fake(48, (24,), bf)), (3, 3.0), (3, 1 << 40), (4, 1),
                    (5, "1"), (6, fake(96, (2, 5, 23))), (6, fake(96, (5, 2, 24))), (6, None), (7, fake(80, (2, 4, 2))), (8, rows8(160, 9, 24)),
                    (8, out), (9, fake(320, (9,), contiguous=False))):
        args = list(good)
        args[at] = bad
        assert c.norm(*args) is NotImplemented, at
    good = [x, x, stats, g, g, 3, 0, out, g, g, None]
    for at, bad in ((0, fake(16, (10, 24))), (1, rows8(160, 11, 24)), (1, fake(16, (2, 5, 25))), (2, None), (3, fake(48, (23,))), (7, fake(96, (2, 5, 24), bf)),
                    (8, None), (9, fake(48, (25,))), (10, fake(320, (9,), cuda=False))):
        args = list(good)
        args[at] = bad
        assert c.norm_backward(*args) is NotImplemented, at
    a, w, out = rows8(64, 6, 40), rows8(128, 9, 40), fake(1024, (6, 9))
    for bad in ((a, rows8(128, 9, 60), None, out), (a, w, fake(512, (8,)), out), (a, w, None, fake(1024, (6, 8))), (a, w, None, fake(1024, (7, 9))),
                (a, w, None, fake(1024, (6, 9), i8)), (list(a), w, None, out), (a, w, None, None),
                ((fake(64, (6, 40), i8), a[1]), (fake(128, (9, 40), i8), w[1]), None, out), ((fake(64, (288,), i8), a[1]), w, None, out)):
        assert c.matmul(*bad) is NotImplemented
    assert not seen
