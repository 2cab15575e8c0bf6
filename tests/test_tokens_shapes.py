"""Outputs of the channels-last operators have the shape of what is written into them, by either route of a call."""
import pytest

from paper_2006_09791_amd import binding as b
from test_tokens_call import call, fake  # noqa: F401  (fixture)

torch = pytest.importorskip("torch")


class Fake(torch.Tensor):
    """A host tensor that says it is on the GPU: what is refused for its shape never gets to be read."""
    is_cuda = True


def test_layout_outputs(call):  # noqa: F811
    c, seen = call
    for out in ((2, 5, 3), (2, 1, 5, 3), (2, 5, 1, 3), (10, 3)):
        assert c.pack(fake(16, (2, 3, 5)), fake(32, out)) == -100
    for out in ((2, 3, 5), (2, 3, 5, 1), (2, 3, 1, 5)):
        assert c.unpack(fake(16, (2, 5, 3)), fake(32, out)) == -101
    assert [a[2:5] for _, a in seen] == [(2, 3, 5)] * 7
    del seen[:]
    for out in ((2, 3, 5), (5, 2, 3), (3, 10), (30,), (1, 10, 3), (5, 6), (30, 1)):
        assert c.pack(fake(16, (2, 3, 5)), fake(32, out)) is NotImplemented
        with pytest.raises(b.GspcError, match="out has shape"):
            b.gspc_pack_channels_last(torch.zeros(2, 3, 5).as_subclass(Fake), out=torch.zeros(out).as_subclass(Fake))
    for out in ((2, 5, 3), (5, 3, 2), (2, 15), (30,), (1, 3, 10)):
        assert c.unpack(fake(16, (2, 5, 3)), fake(32, out)) is NotImplemented
        with pytest.raises(b.GspcError, match="out has shape"):
            b.gspc_unpack_channels_last(torch.zeros(2, 5, 3).as_subclass(Fake), out=torch.zeros(out).as_subclass(Fake))
    assert not seen


def test_norm_tensors_of_another_shape_are_left_to_the_general_route(call):  # noqa: F811
    """Which refuses them: pixels in another order are another image."""
    c, seen = call
    x, stats, v = fake(16, (2, 3, 4, 24)), fake(80, (2, 3, 2)), fake(48, (24,))
    same, turned, flat = fake(96, (2, 3, 4, 24)), fake(96, (2, 4, 3, 24)), fake(96, (2, 12, 24))
    norm = lambda x, y: c.norm(x, v, v, 3, 1e-5, 0, y, None, None, None)  # noqa: E731
    back = lambda dy, x, dx: c.norm_backward(dy, x, stats, v, v, 3, 0, dx, v, v, None)  # noqa: E731
    assert norm(x, same) == -104 and back(x, same, same) == -105 and len(seen) == 2
    for other in (turned, flat, fake(96, (2, 3, 2, 2, 24))):
        assert norm(x, other) is back(x, other, same) is back(x, same, other) is NotImplemented
    assert len(seen) == 2


def test_pairs_may_be_lists():
    """8-bit rows as a list of two, outputs given or not: what is wrong with host tensors is that they are not on the GPU."""
    x, pair = torch.zeros(2, 3, 16), [torch.zeros(6, 16, dtype=torch.int8), torch.zeros(6)]
    for c in (lambda: b.gspc_group_norm(x, None, None, 4, out=pair), lambda: b.gspc_group_norm(x, None, None, 4, saved=pair),
              lambda: b.gspc_group_norm_backward(x, pair, torch.zeros(2, 4, 2), None, None, 4),
              lambda: b.gspc_quantize_rows(x, out=pair), lambda: b.gspc_dequantize_rows(pair, 16), lambda: b.gspc_matmul_i8(pair, pair)):
        with pytest.raises(b.GspcError, match="GPU"):
            c()
