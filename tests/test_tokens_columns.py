"""How many columns of two operands of 8-bit rows are summed: the pitch, or the length that the caller names."""
import pytest

from paper_2006_09791_amd import binding as b
from test_tokens_call import call, fake, rows8  # noqa: F401  (fixture)

torch = pytest.importorskip("torch")


def test_named_length_arrives(call):  # noqa: F811
    c, seen = call
    a, w, out = rows8(64, 6, 133144), rows8(128, 9, 133144), fake(1024, (6, 9))
    assert c.matmul(a, w, None, out, 133144) == c.matmul(a, w, None, out, 133137) == c.matmul(a, w, None, out, None) == -106
    assert [args[7] for _, args in seen] == [133144, 133137, 133152]
    del seen[:]
    for cols in (133136, 133153, 0, -5, 40.0, "40", 1 << 31, 1 << 40):
        assert c.matmul(a, w, None, out, cols) is NotImplemented
    assert c.matmul(a, w, None, out, 133144, 1) is NotImplemented and not seen


def test_length_that_is_not_the_operands():
    host = lambda rows, cols: (torch.zeros(rows, b.gspc_rows8_pitch(cols), dtype=torch.int8), torch.zeros(rows))  # noqa: E731
    for cols in (320, 337, 16):
        with pytest.raises(b.GspcError, match=f"rows of {cols} values"):
            b.gspc_matmul_i8(host(2, 333), host(3, 333), cols=cols)
    with pytest.raises(b.GspcError, match="GPU"):               # (the length is not what is wrong)
        b.gspc_matmul_i8(host(2, 333), host(3, 333), cols=333)
