"""Channels-last operators at counts that pass what one launch may have: many small images, one very large plane."""
import pytest

from test_gpu_parity import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
MANY = 17_000_000               # images: in blocks of 256 threads more than 2^32 threads


@pytest.mark.parametrize("C,P", [(8, 8), (3, 2)])
def test_layout_of_many_images(gpu, C, P):
    torch, b = gpu
    x = torch.randn(MANY, C, P, device="cuda").bfloat16()
    y = b.gspc_pack_channels_last(x)
    assert torch.equal(y, x.transpose(1, 2))
    z = b.gspc_unpack_channels_last(y, dtype=b.GSPC_BF16)
    assert torch.equal(z, x)


def test_layout_of_one_large_plane(gpu):
    """2^24 + 1 tiles of one plane: a number made of its place in each of its elements."""
    torch, b = gpu
    C, P, piece = 8, (1 << 30) + 1, 1 << 26
    x = torch.empty(1, C, P, dtype=torch.int16, device="cuda")
    number = lambda c, at: ((torch.arange(at, min(at + piece, P), device="cuda") * 40503 + c * 977) & 0x3fff).short()  # noqa: E731
    for c in range(C):
        for at in range(0, P, piece):
            x[0, c, at:at + piece] = number(c, at)
    y = b.gspc_pack_channels_last(x.view(torch.bfloat16)).view(torch.int16)
    for c in range(C):
        for at in range(0, P, piece):
            assert torch.equal(y[0, at:at + piece, c], number(c, at)), (c, at)
