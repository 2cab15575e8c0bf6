"""Gradient of group norm with ReLU where no value lies near the jump: every element of dx has to be right.

Near means within 16 u (1 + |xh| + |mean| rstd) (|gamma| + |beta|) of zero, u = 2^-24: what rounding may move z by.  Inputs come from the first seed
that has none."""
import numpy as np
import pytest

from test_gpu_parity import gpu  # noqa: F401  (fixture)
from test_gpu_tokens import B, U, dev, grad64, host, norm64, norm_inputs

pytestmark = pytest.mark.gpu


def inputs(torch, shape, src):
    N, P, C, groups = shape
    for seed in range(200):
        x, gamma, beta = norm_inputs(N, P, C, 1000 + seed)
        xd = dev(torch, x, getattr(torch, src))
        xh, z, mean, rstd, _ = norm64(host(xd), gamma.astype(float), beta.astype(float), groups, 1e-5)
        near = np.abs(z) <= 16 * U * (1 + np.abs(xh) + np.abs(mean) * rstd) * (np.abs(gamma) + np.abs(beta))
        if not near.any():
            return xd, gamma, beta, seed
    raise AssertionError("no seed without a value near the jump")


@pytest.mark.parametrize("shape", [(2, 17, 6, 3), (5, 63, 60, 3), (2, 49, 512, 32), (1, 12544, 16, 2), (4, 200, 130, 13), (1, 7, 2050, 2), (3, 50, 96, 96)], ids=str)
@pytest.mark.parametrize("src,grad", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "bfloat16")])
def test_relu_gradient_away_from_the_jump(gpu, shape, src, grad):
    torch, b = gpu
    N, P, C, groups = shape
    xd, gamma, beta, seed = inputs(torch, shape, src)
    dyd = dev(torch, np.random.default_rng(seed).standard_normal((N, P, C)).astype(np.float32), getattr(torch, grad))
    gd, bd, st = dev(torch, gamma), dev(torch, beta), torch.empty(N, groups, 2, device="cuda")
    b.gspc_group_norm(xd, gd, bd, groups, act=b.ACT_RELU, stats=st)
    dx, dgamma, dbeta, size, size_g, size_b, xh, shift = grad64(host(dyd), host(xd), host(st), gamma.astype(float), beta.astype(float), groups, 1)
    got = b.gspc_group_norm_backward(dyd, xd, st, gd, bd, groups, b.ACT_RELU)
    tol = 256 * U * size * (1 + np.abs(xh) + np.abs(shift)) + (B * np.abs(dx) if grad == "bfloat16" else 0) + 1e-30
    rel = 1 + np.abs(shift).max()
    assert (np.abs(host(got[0]) - dx) <= tol).all(), np.max(np.abs(host(got[0]) - dx) / tol)
    assert (np.abs(host(got[1]) - dgamma) <= 256 * U * rel * size_g + 1e-30).all()
    assert (np.abs(host(got[2]) - dbeta) <= 256 * U * rel * size_b + 1e-30).all()
