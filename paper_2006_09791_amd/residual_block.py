"""Residual blocks of pointwise layers on tokens, in 8-bit floating point, as a network answers with them and as it is trained: the stream is
normalised and activated, a layer's product is normalised, gated, thinned by dropout and added to the stream.

    x' = scale x + gate * dropout(post(z w^T)),    z = act(pre(x)),    block after block

    python -m paper_2006_09791_amd.residual_block [--images 64] [--pixels 14] [--channels 512] [--blocks 4] [--drop 0.1]
"""
import argparse
import math
import time

from . import binding as b


class ResidualBlocks:
    """weights [C, C], gates, post_gammas, pre_gammas [C]: lists of fp32 tensors on the GPU, one for each block.  What a pass makes for itself and
    drops at its end belongs to the library's stream (binding._empty)."""

    def __init__(self, weights, gates, post_gammas, pre_gammas, scale=1.0, drop=0.0, seed=0, norm=b.NORM_RMS, act=b.ACT_SILU, eps=1e-5):
        self.weights, self.gates, self.post, self.pre = weights, gates, post_gammas, pre_gammas
        self.scale, self.drop, self.seed, self.norm, self.act, self.eps = scale, drop, seed, norm, act, eps

    def weight_rows(self):
        """The weights as they are now, as 8-bit float rows: for answers of weights that stay, once."""
        return [b.gspc_quantize_rows_f8(w) for w in self.weights]

    def _before(self, k):
        """The norm in front of block k, or none behind the last."""
        if k == len(self.weights):
            return {"eps": self.eps}
        return {"pre": self.norm, "pre_gamma": self.pre[k], "act": self.act, "eps": self.eps}

    def _block(self, k, step):
        """What adds block k to the stream, and normalises it for the next.  (A block's dropout is a call of its own: the upper half of the offset.)"""
        return {"gate": self.gates[k], "post": self.norm, "post_gamma": self.post[k], "scale": self.scale, **self._before(k + 1),
                **({"drop": self.drop, "seed": self.seed, "offset": k << 32, "step": step} if step is not None else {})}

    def answer(self, x, rows8=None):
        """x [N, P, C] -> [N, P, C], of its type.  rows8: what weight_rows returned, while the weights are those of then; without it each answer
        writes them anew."""
        if rows8 is not None and len(rows8) != len(self.weights):
            raise b.GspcError(-5, f"rows of {len(rows8)} weights, blocks {len(self.weights)}")
        _, z = b.gspc_residual_norm(x, dtype=b.GSPC_F8, **self._before(0))
        for k, w in enumerate(self.weight_rows() if rows8 is None else rows8):
            h = b.gspc_matmul_f8(z, w).view(x.shape)
            # (the stream is written in place from the second block on: x itself stays)
            x, z = b.gspc_residual_norm(x, h, xo=x if k else None, dtype=b.GSPC_F8, **self._block(k, None))
        return x

    def train(self, x, dy, step):
        """The pass over x [N, P, C] and back from dy, the gradient of its output: (output, dx, [gradients of each block: ResidualGradients of the sum,
        and the weight's]), then the first norm's.  step: an int64 tensor of one value, another one for each pass: dropout's calls are told
        apart by it (in a captured graph too)."""
        import torch
        rows, C = x.numel() // x.shape[-1], x.shape[-1]
        kept, forms = [], []
        stats = b._empty((rows, 4), torch.float32, x.device)
        xo, z = b.gspc_residual_norm(x, stats=stats, **self._before(0))
        first = stats
        for k, w in enumerate(self.weights):
            tokens, columns = b.gspc_quantize_rows_f8(z, which=b.F8_BOTH)
            w_rows, w_columns = b.gspc_quantize_rows_f8(w, which=b.F8_BOTH)     # (another weight in each step)
            h = b.gspc_matmul_f8(tokens, w_rows).view(x.shape)
            stats = b._empty((rows, 4), torch.float32, x.device)
            xo, z = b.gspc_residual_norm(xo, h, stats=stats, **self._block(k, step))
            kept.append((xo, h, stats))
            forms.append((columns, w_columns))
        out, dz, grads = xo, None, []
        for k in reversed(range(len(self.weights))):
            xo, h, stats = kept[k]
            settings = {name: v for name, v in self._block(k, step).items() if name != "eps"}
            g = b.gspc_residual_norm_backward(dz, dy, xo, h, stats, **settings)
            rows8, columns8 = b.gspc_quantize_rows_f8(g.dh, which=b.F8_BOTH)
            columns, w_columns = forms[k]
            dz = b.gspc_matmul_f8(rows8, w_columns).view(x.shape)
            grads.append((g, b.gspc_matmul_f8(columns8, columns, dtype=b.GSPC_F32)))
            dy = g.dx
        settings = {name: v for name, v in self._before(0).items() if name != "eps"}
        g = b.gspc_residual_norm_backward(dz, dy, x, None, first, **settings)
        return out, g.dx, grads[::-1], g


def random_blocks(C, blocks, drop=0.0, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    each = lambda f: [f() for _ in range(blocks)]  # noqa: E731
    return ResidualBlocks(each(lambda: r(C, C) * math.sqrt(2 / C)), each(lambda: 0.5 + 0.1 * r(C)), each(lambda: 1 + 0.2 * r(C)),
                          each(lambda: 1 + 0.2 * r(C)), drop=drop, seed=seed)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--images", type=int, default=64)
    ap.add_argument("--pixels", type=int, default=14)
    ap.add_argument("--channels", type=int, default=512)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--drop", type=float, default=0.1)
    ap.add_argument("--passes", type=int, default=50)
    a = ap.parse_args()
    import torch
    b.gspc_set_stream()
    net = random_blocks(a.channels, a.blocks, a.drop)
    rows8 = net.weight_rows()
    x = torch.randn(a.images, a.pixels * a.pixels, a.channels, device="cuda").bfloat16()
    dy, step = torch.randn_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")

    def train():
        net.train(x, dy, step)
        step.add_(1)
    for name, call in (("answer", lambda: net.answer(x, rows8)), ("train", train)):
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
