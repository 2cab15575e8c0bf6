"""A block of a grouped network with its pointwise layer in 8 bits: a grouped 3x3 convolution, group norm with SiLU on
channels-last tokens that writes 8-bit rows, and the product with 8-bit weights, back to planes for the next grouped
convolution.  And one training pass through the norm, which keeps 8-bit rows of its input for the gradient.

    python -m paper_2006_09791_amd.token_block [--images 64] [--channels 128] [--pixels 28] [--groups 4] [--filters 256]
"""
import argparse
import math
import time

from . import binding as b


class TokenBlock:
    """weight [C, C/groups, 3, 3], gamma and beta [C], pointwise [filters, C]: fp32 tensors on the GPU.  What a pass makes for itself and drops
    at its end belongs to the library's stream (binding._empty): torch gives it to no other stream's work before that stream is done."""

    def __init__(self, weight, gamma, beta, pointwise, conv_groups, norm_groups, eps=1e-5):
        self.C, self.conv_groups, self.norm_groups, self.eps = weight.shape[0], conv_groups, norm_groups, eps
        self.packed = b.gspc_pack_weights(weight, conv_groups)
        self.gamma, self.beta = gamma, beta
        self.pointwise = b.gspc_quantize_rows(pointwise)        # once: a scale for each filter
        self.filters = pointwise.shape[0]

    def tokens(self, x):
        """x [N, C, H, W] fp32 -> what the convolution leaves, as bf16 tokens [N, H * W, C]."""
        import torch
        N, C, H, W = x.shape
        y = b._empty((N, C, H, W), torch.float32, x.device)
        b.gspc_conv2d_grouped(x, self.packed, N, C, H, W, C, 3, 3, 1, 1, self.conv_groups, output=y)
        return b.gspc_pack_channels_last(y)

    def answer(self, x):
        """x [N, C, H, W] fp32 -> [N, filters, H, W] fp32."""
        N, _, H, W = x.shape
        rows8 = b.gspc_group_norm(self.tokens(x), self.gamma, self.beta, self.norm_groups, self.eps, b.ACT_SILU, dtype=b.GSPC_I8)
        out = b.gspc_matmul_i8(rows8, self.pointwise)
        return b.gspc_unpack_channels_last(out.view(N, H * W, self.filters)).view(N, self.filters, H, W)

    def train(self, tokens, dy):
        """The norm's pass over tokens [N, P, C] and back: (y, dx, dgamma, dbeta).  Between the two only 8-bit rows of the tokens and
        two numbers for each group are kept."""
        import torch
        N, P, C = tokens.shape
        stats = b._empty((N, self.norm_groups, 2), torch.float32, tokens.device)
        saved = b._new_rows8(N * P, C, tokens.device)
        y = b.gspc_group_norm(tokens, self.gamma, self.beta, self.norm_groups, self.eps, b.ACT_SILU, stats=stats, saved=saved)
        return (y, *b.gspc_group_norm_backward(dy, saved, stats, self.gamma, self.beta, self.norm_groups, b.ACT_SILU))


def random_block(C, filters, conv_groups, norm_groups, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    return TokenBlock(r(C, C // conv_groups, 3, 3) * math.sqrt(2 / (9 * C // conv_groups)), 1 + 0.2 * r(C), 0.2 * r(C),
                      r(filters, C) * math.sqrt(2 / C), conv_groups, norm_groups)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--images", type=int, default=64)
    ap.add_argument("--channels", type=int, default=128)
    ap.add_argument("--pixels", type=int, default=28)
    ap.add_argument("--groups", type=int, default=4, help="of the convolution")
    ap.add_argument("--norm-groups", type=int, default=32)
    ap.add_argument("--filters", type=int, default=256)
    ap.add_argument("--passes", type=int, default=50)
    a = ap.parse_args()
    import torch
    b.gspc_set_stream()
    block = random_block(a.channels, a.filters, a.groups, a.norm_groups)
    x = torch.randn(a.images, a.channels, a.pixels, a.pixels, device="cuda")
    tokens = block.tokens(x)
    dy = torch.randn_like(tokens)
    for name, call in (("answer", lambda: block.answer(x)), ("train", lambda: block.train(tokens, dy))):
        for _ in range(5):
            call()
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(a.passes):
            call()
        torch.cuda.synchronize()
        print(f"{name}: {(time.perf_counter() - began) / a.passes * 1e6:.1f} us a pass")


if __name__ == "__main__":
    main()
