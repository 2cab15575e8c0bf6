"""Dropout on the GPU against its definition: which values are dropped has to be equal, what is kept is one product, rounded once."""
import numpy as np
import pytest

from block_reference import dropout_factors, on_side_stream
from test_gpu_parity import gpu  # noqa: F401  (fixture)
from test_gpu_tokens import dev, strided

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (130, 9), (7, 64), (65, 333), (5, 4104), (1000, 3), (257, 512)])
@pytest.mark.parametrize("drop", [0.0, 0.1, 0.5, 2.0 ** -16, 0.99999, 1.0])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_dropout(gpu, rows, cols, drop, dtype):
    torch, b = gpu
    rng = np.random.default_rng(rows + cols)
    x = dev(torch, rng.standard_normal((rows, cols)).astype(np.float32), getattr(torch, dtype))
    seed, offset = int(rng.integers(1 << 63)) * 2 + 1, int(rng.integers(1 << 62))
    m = dropout_factors(rows, cols, drop, seed, offset).astype(np.float32)      # (the factor is an fp32 number)
    want = torch.from_numpy(x.float().cpu().numpy() * m).to(x.dtype)
    assert torch.equal(b.gspc_dropout(x, drop, seed, offset).cpu(), want)
    _, view = strided(torch, x, 6)
    wide = torch.full((rows + 2, cols + 6), 5.0, dtype=x.dtype, device="cuda")
    b.gspc_dropout(view, drop, seed, offset, out=wide[1:-1, 3:-3])
    assert torch.equal(wide[1:-1, 3:-3].cpu(), want)
    wide[1:-1, 3:-3] = 5.0
    assert bool((wide == 5.0).all())
    assert b.gspc_dropout(x, drop, seed, offset, out=x) is x and torch.equal(x.cpu(), want)     # in place


def test_published_numbers(gpu):
    """The generator's published values of counter and key zero, through the kernel: thresholds just at and above each 16-bit half tell it."""
    torch, b = gpu
    words = 0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8
    x = torch.ones(1, 8, device="cuda")
    for k, half in enumerate(h for w in words for h in (w & 0xffff, w >> 16)):
        assert b.gspc_dropout(x, half / 65536, 0)[0, k] > 0 and b.gspc_dropout(x, (half + 1) / 65536, 0)[0, k] == 0


def test_what_is_dropped_is_zero_whatever_it_was(gpu):
    torch, b = gpu
    x = torch.full((50, 40), float("nan"), device="cuda")
    x[::2] = float("inf")
    m = torch.from_numpy(dropout_factors(50, 40, 0.4, 5, 6)).cuda()
    y = b.gspc_dropout(x, 0.4, 5, 6)
    assert bool((y[m == 0] == 0).all()) and bool(y[1::2][m[1::2] > 0].isnan().all()) and bool((y[::2][m[::2] > 0] == float("inf")).all())


def test_masks_differ_and_are_balanced(gpu):
    """Another seed, offset, row or vector gives other numbers.  Of n values at p, the number dropped is within 6 deviations sqrt(n p (1 - p))."""
    torch, b = gpu
    x = torch.ones(2000, 512, device="cuda")
    n = x.numel()
    masks = [b.gspc_dropout(x, 0.3, s, o) > 0 for s, o in ((1, 0), (2, 0), (1, 1), (1, 1 << 32), (1 + (1 << 32), 0), ((1 << 64) - 1, (1 << 64) - 1))]
    for i, m in enumerate(masks):
        assert abs(int(m.sum()) - 0.7 * n) < 6 * (n * 0.21) ** 0.5
        for other in masks[:i]:                 # both keep with 0.49
            assert abs(int((m & other).sum()) - 0.49 * n) < 6 * (n * 0.49 * 0.51) ** 0.5
    m = masks[0].float() - 0.7
    for shifted in (m.roll(1, 0), m.roll(1, 1), m.roll(8, 1)):
        assert abs(float((m * shifted).sum())) < 6 * 0.21 * n ** 0.5


def test_dropout_in_a_replayed_graph_takes_its_offset_from_a_tensor(gpu):
    torch, b = gpu
    x, step = torch.randn(130, 100, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    with on_side_stream(torch, b) as s:
        b.gspc_dropout(x, 0.5, 9, 4, step)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            y = b.gspc_dropout(x, 0.5, 9, 4, step)
            step += 1
        for k in range(4):
            graph.replay()
            torch.cuda.synchronize()
            want = b.gspc_dropout(x, 0.5, 9, 4 + k)
            s.synchronize()
            assert torch.equal(y, want), k
        step.fill_(-1)                          # (64 bits that wrap)
        torch.cuda.synchronize()
        got = b.gspc_dropout(x, 0.5, 9, 4, step)
        s.synchronize()
        assert torch.equal(got, b.gspc_dropout(x, 0.5, 9, 3))


def test_dropout_past_32_bits(gpu):
    torch, b = gpu
    C = 512
    rows = (1 << 32) // C + 4096
    x = torch.ones(rows, C, dtype=torch.bfloat16, device="cuda")
    b.gspc_dropout(x, 0.5, 3, 8, out=x)
    for at in (0, 1 << 21, rows - 100):
        m = dropout_factors(np.arange(at, at + 100), C, 0.5, 3, 8)
        assert np.array_equal(x[at:at + 100].float().cpu().numpy(), m)
