"""The block that runs the channels-last operators together, against the oracle's convolution and the definitions in 64 bits.

Tolerance on the whole (2-norm of the difference over that of the result): rounding a row to 8 bits is off by a uniform step of
max / 127, sqrt(1/12) of it in the mean square; with max below 5 times the row's root mean square that is 5 / 127 / 3.5 = 1.2 % of
it, for tokens and weights alike, 1.6 % together; tokens in bf16 add 0.2 %, products in bf16 another.  3 % is allowed."""
import numpy as np
import pytest

import oracle
from test_gpu_parity import gpu  # noqa: F401  (fixture)
from test_gpu_tokens import act64, grad64, norm64

pytestmark = pytest.mark.gpu


def far(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("N,C,H,W,conv_groups,norm_groups,filters", [(2, 32, 14, 14, 4, 8, 64), (3, 48, 9, 7, 3, 6, 33), (1, 64, 8, 8, 64, 32, 10)])
def test_block(gpu, N, C, H, W, conv_groups, norm_groups, filters):
    torch, b = gpu
    from paper_2006_09791_amd import token_block
    g = torch.Generator(device="cuda").manual_seed(N + C)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    weight, gamma, beta, pointwise = r(C, C // conv_groups, 3, 3), 1 + 0.2 * r(C), 0.2 * r(C), r(filters, C)
    block = token_block.TokenBlock(weight, gamma, beta, pointwise, conv_groups, norm_groups)
    x, host = r(N, C, H, W), lambda t: t.double().cpu().numpy()
    out = block.answer(x)
    assert out.shape == (N, filters, H, W) and out.dtype == torch.float32
    y = oracle.conv2d_grouped(x.cpu().numpy(), weight.cpu().numpy(), 1, 1, conv_groups, threads=4)
    t = np.asarray(y, np.float64).reshape(N, C, H * W).transpose(0, 2, 1)
    z = act64(norm64(t, host(gamma), host(beta), norm_groups, 1e-5)[1], 2)
    want = (z @ host(pointwise).T).transpose(0, 2, 1).reshape(out.shape)
    assert far(host(out), want) < 0.03

    tokens = block.tokens(x)
    assert far(host(tokens), t) < 0.004                       # one rounding to bf16
    dy = r(N, H * W, C).bfloat16()
    y2, dx, dgamma, dbeta = block.train(tokens, dy)
    t = host(tokens)
    _, z, _, _, stats = norm64(t, host(gamma), host(beta), norm_groups, 1e-5)
    assert far(host(y2), act64(z, 2)) < 0.004
    q = b.gspc_quantize_rows(tokens)
    kept = (host(q[0])[:, :C] * host(q[1])[:, None]).reshape(t.shape)
    want = grad64(host(dy), kept, stats, host(gamma), host(beta), norm_groups, 2)
    for got, w, tol in ((dx, want[0], 0.004), (dgamma, want[1], 1e-4), (dbeta, want[2], 1e-4)):
        assert far(host(got), w) < tol
    # and what 8 bits cost against the gradient of the tokens themselves: the two steps' error, as above
    want = grad64(host(dy), t, stats, host(gamma), host(beta), norm_groups, 2)
    assert far(host(dx), want[0]) < 0.03 and far(host(dgamma), want[1]) < 0.03


def test_command_prints_both_passes(gpu, capsys, monkeypatch):
    from paper_2006_09791_amd import token_block
    monkeypatch.setattr("sys.argv", ["token_block", "--images", "2", "--channels", "32", "--pixels", "7", "--norm-groups", "8", "--filters", "40",
                                     "--passes", "2"])
    token_block.main()
    text = capsys.readouterr().out
    assert "answer:" in text and "train:" in text
