"""What dropout drops is 0 whatever it was, in the gradient too: values that are no number, where they are dropped, have no say in what is added up over
tokens."""
import pytest

from block_reference import dropout_factors
from test_gpu_parity import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
DROP, SEED, OFFSET = 0.4, 11, 12


def tensors(torch, rows, C, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + C)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    return [r(rows, C).to(dtype) for _ in range(4)] + [1 + 0.2 * r(C) for _ in range(4)]


# a few lanes a token, a ragged row, a wave, several, and as many as there are
SIZES = [(40, 5), (40, 24), (40, 130), (36, 512), (20, 1000), (12, 4104), (12, 8192)]


@pytest.mark.parametrize("rows,C", SIZES)
@pytest.mark.parametrize("gates", ["one", "each", "some"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_dropped_infinities_without_a_norm(gpu, rows, C, gates, dtype):
    """Bit by bit the gradient of a tensor that has zeros there."""
    torch, b = gpu
    x, h, dz, dxo, g1, b1, g2, b2 = tensors(torch, rows, C, getattr(torch, dtype))
    n = {"one": 1, "each": rows, "some": 4}[gates]
    kw = dict(gate=torch.randn(n, C, device="cuda"), pre=b.NORM_LAYER, pre_gamma=g2, pre_beta=b2, act=b.ACT_SILU, drop=DROP, seed=SEED, offset=OFFSET)
    m = torch.from_numpy(dropout_factors(rows, C, DROP, SEED, OFFSET) == 0).cuda()
    zero = torch.where(m, torch.zeros_like(h), h)
    stats, want_stats = (torch.empty(rows, 4, device="cuda") for _ in range(2))
    xo, z = b.gspc_residual_norm(x, zero, stats=want_stats, **kw)
    want = b.gspc_residual_norm_backward(dz, dxo, xo, zero, want_stats, **kw)
    for what in (float("inf"), float("-inf"), float("nan")):
        bad = torch.where(m, torch.full_like(h, what), h)
        got_xo, got_z = b.gspc_residual_norm(x, bad, stats=stats, **kw)
        assert torch.equal(got_xo, xo) and torch.equal(got_z, z) and torch.equal(stats, want_stats)
        got = b.gspc_residual_norm_backward(dz, dxo, got_xo, bad, stats, **kw)
        for name in ("dx", "dh", "dgate", "dpre_gamma", "dpre_beta"):
            assert torch.equal(getattr(got, name), getattr(want, name)), (name, what)
    everything = b.gspc_residual_norm_backward(dz, dxo, xo, torch.full_like(h, float("nan")), want_stats, **{**kw, "drop": 1.0})
    assert bool((everything.dgate == 0).all()) and bool((everything.dh == 0).all())


@pytest.mark.parametrize("rows,C", SIZES)
@pytest.mark.parametrize("post", [1, 2])
@pytest.mark.parametrize("gates", [1, 4])
def test_a_normalised_token_that_is_no_number(gpu, rows, C, post, gates):
    """All of such a token is no number: the channels that it keeps make their sums none, the others' sums are, bit by bit, those of the token as it was,
    which adds zeros to them."""
    torch, b = gpu
    x, h, _, dxo, g1, b1, _, _ = tensors(torch, rows, C, torch.float32)
    gate = 1 + 0.1 * torch.randn(gates, C, device="cuda")
    kw = dict(gate=gate, post=post, post_gamma=g1, post_beta=b1, drop=DROP, seed=SEED, offset=OFFSET)
    m = torch.from_numpy(dropout_factors(rows, C, DROP, SEED, OFFSET) == 0).cuda()
    stats = torch.empty(rows, 4, device="cuda")
    xo, _ = b.gspc_residual_norm(x, h, stats=stats, **kw)
    want = b.gspc_residual_norm_backward(None, dxo, xo, h, stats, **kw)
    t = rows // 2
    h[t] = float("nan")
    xo, _ = b.gspc_residual_norm(x, h, stats=stats, **kw)
    got = b.gspc_residual_norm_backward(None, dxo, xo, h, stats, **kw)
    dropped = m[t]
    assert torch.equal(got.dx, want.dx)
    own = t // (rows // gates)
    for g, w in ((got.dpost_gamma, want.dpost_gamma), (got.dgate[own], want.dgate[own])):
        assert bool(g[~dropped].isnan().all()) and torch.equal(g[dropped], w[dropped])
    assert torch.equal(got.dpost_beta, want.dpost_beta)         # (its terms hold no h)
