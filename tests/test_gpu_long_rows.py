"""Rows of more than 2^32 bytes (fp32, 2^30 columns and some): at both ends and around 2^32 bytes their columns get, bit by bit, what a short row of the same
values gets by itself."""
import numpy as np
import pytest

from block_reference import philox
from test_gpu_parity import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
LENGTHS = [(1 << 30) + 136, (1 << 30) + 333]        # whole eights, and not
SEED, OFFSET = 3, 8


def pieces(C):
    """[first, last) of some stretches that begin on a block of 128 columns."""
    for at in (0, (1 << 29) - 512, (1 << 30) - 512, (1 << 30) + 128):
        yield at, min(at + 1024, C)


def factors(first, last):
    """Dropout's, of row 0 at the probability 1/2."""
    vec = np.arange(first // 8, (last + 7) // 8)
    words = philox((vec, np.zeros_like(vec), np.full_like(vec, OFFSET), np.zeros_like(vec)), SEED)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xffff), w >> np.uint64(16))], 1).reshape(-1)
    return np.where(halves >= 32768, 2.0, 0.0)[:last - first]


@pytest.mark.parametrize("C", LENGTHS)
def test_dropout(gpu, C):
    torch, b = gpu
    x = torch.randn(1, C, device="cuda")
    y = b.gspc_dropout(x, 0.5, SEED, OFFSET)
    want = [x[0, s:e] * torch.from_numpy(factors(s, e)).float().cuda() for s, e in pieces(C)]
    assert all(torch.equal(y[0, s:e], w) for (s, e), w in zip(pieces(C), want))
    dropped = int((y == 0).sum())
    assert abs(dropped - C / 2) < 6 * (C / 4) ** 0.5
    b.gspc_dropout(x, 0.5, SEED, OFFSET, out=x)             # in place
    assert torch.equal(x, y)


@pytest.mark.parametrize("C", LENGTHS)
def test_8_bit_float_rows_and_back(gpu, C):
    torch, b = gpu
    x = torch.randn(1, C, device="cuda")
    q, scale = b.gspc_quantize_rows_f8(x)
    back = b.gspc_dequantize_rows_f8((q, scale), C)
    for s, e in pieces(C):
        short = x[:, s:e].contiguous()
        want = b.gspc_quantize_rows_f8(short)
        blocks = (e - s + 127) // 128
        assert torch.equal(q[:, s:s + blocks * 128].view(torch.uint8), want[0].view(torch.uint8))
        assert torch.equal(scale[:, s // 128:s // 128 + blocks], want[1][:, :blocks])
        assert torch.equal(back[:, s:e], b.gspc_dequantize_rows_f8(want, e - s))


def test_8_bit_float_rows_along_the_columns(gpu):
    """One value a row of the transpose: 128 bytes for each of 2^30 columns."""
    torch, b = gpu
    C = LENGTHS[1]
    if torch.cuda.mem_get_info()[0] < 200 << 30:
        pytest.skip("150 GB of memory are needed")
    x = torch.randn(1, C, device="cuda")
    q, scale = b.gspc_quantize_rows_f8(x, which=b.F8_COLUMNS)
    for s, e in pieces(C):
        want = b.gspc_quantize_rows_f8(x[:, s:e].contiguous(), which=b.F8_COLUMNS)
        assert torch.equal(q[s:e].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(scale[s:e], want[1])
    del q, scale
    torch.cuda.empty_cache()
