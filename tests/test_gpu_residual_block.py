"""The residual blocks that run the operators together, for answers and a training step, against the same network in 64 bits.

Tolerances on the whole (2-norm of the difference over that of the result).  Rounding to e4m3 is off by a uniform step of 1/8 of the power of two below
the value, sqrt(1/12) of it in the mean square: 0.125 / 3.46 / 1.44 = 2.5 % of it, for both operands of a product 3.5 %.  x' holds the stream, which is
not rounded to 8 bits, and half of it: less than 3.5 % after any number of blocks that each add as much anew; z, which is its norm, as much, and
through SiLU's slope, at most 1.1, 4 %.  A gradient goes through as many products back, each 3.5 % with what z is off: with two blocks sqrt(4) 4 % = 8 %.
5 and 12 % are allowed."""
import numpy as np
import pytest

from block_reference import backward64, dropout_factors, forward64, on_side_stream
from test_gpu_parity import gpu  # noqa: F401  (fixture)
from test_gpu_token_block import far
from test_gpu_tokens import host

pytestmark = pytest.mark.gpu


def network64(net, x, dy, offsets):
    """(output, dx, [(gradients of a block), ...]) in 64 bits; offsets: of each block's dropout, or None without."""
    rows, C = x.shape
    none = dict.fromkeys(("post_gamma", "post_beta", "pre_gamma", "pre_beta", "gate", "mask"))
    L = len(net.weights)

    def settings(k):
        before = {} if k + 1 == L else {"pre_gamma": host(net.pre[k + 1])}
        mask = None if offsets is None else dropout_factors(rows, C, net.drop, net.seed, offsets[k])
        return {**none, "post": net.norm, "post_gamma": host(net.post[k]), "gate": host(net.gates[k])[None], "pre": net.norm if before else 0,
                "act": net.act if before else 0, "scale": net.scale, "eps": net.eps, "mask": mask, **before}
    start = {**none, "post": 0, "pre": net.norm, "pre_gamma": host(net.pre[0]), "act": net.act, "scale": 1.0, "eps": net.eps}
    f = forward64(start, x, None)
    kept, zs = [], [f["z"]]
    first, xo = f["stats"], x
    for k in range(L):
        h = zs[-1] @ host(net.weights[k]).T
        f = forward64(settings(k), xo, h)
        xo = f["xo"]
        kept.append((xo, h, f["stats"]))
        zs.append(f["z"])
    dz, grads = None, []
    for k in reversed(range(L)):
        g = {n: v[0] for n, v in backward64(settings(k), dz, dy, *kept[k]).items()}
        g["weight"] = g["dh"].T @ zs[k]
        dz, dy = g["dh"] @ host(net.weights[k]), g["dx"]
        grads.append(g)
    g = {n: v[0] for n, v in backward64(start, dz, dy, x, None, first).items()}
    return xo, g["dx"], grads[::-1], g


@pytest.mark.parametrize("N,P,C,drop", [(2, 49, 128, 0.0), (3, 37, 200, 0.25), (1, 400, 512, 0.1)])
@pytest.mark.parametrize("norm", [1, 2])
def test_two_blocks(gpu, N, P, C, drop, norm):
    torch, b = gpu
    from paper_2006_09791_amd import residual_block
    net = residual_block.random_blocks(C, 2, drop, seed=N + C)
    net.norm = norm
    g = torch.Generator(device="cuda").manual_seed(C)
    x, dy = (torch.randn(N, P, C, device="cuda", generator=g).bfloat16() for _ in range(2))
    keep = x.clone()
    rows = N * P
    flat = lambda t: host(t).reshape(rows, C)  # noqa: E731
    want = network64(net, flat(x), flat(dy), None)
    out = net.answer(x)
    assert out.shape == x.shape and out.dtype == x.dtype and far(flat(out), want[0]) < 0.05
    step = torch.full((1,), 7, dtype=torch.int64, device="cuda")
    out, dx, grads, first = net.train(x, dy, step)
    want = network64(net, flat(x), flat(dy), [7, (1 << 32) + 7] if drop else None)
    assert torch.equal(x, keep)
    assert far(flat(out), want[0]) < 0.05 and far(flat(dx), want[1]) < 0.12
    assert far(host(first.dpre_gamma), want[3]["dpre_gamma"]) < 0.12
    for (got, weight), w in zip(grads, want[2]):
        assert far(host(weight), w["weight"]) < 0.12
        assert far(host(got.dpost_gamma), w["dpost_gamma"]) < 0.12 and far(host(got.dgate), w["dgate"][0]) < 0.12
    assert grads[1][0].dpre_gamma is None                     # (no norm behind the last block)


def test_training_step_in_a_replayed_graph(gpu):
    """Captured, with an eager pass alive; replays with other inputs, weights and masks give what an eager pass gives."""
    torch, b = gpu
    from paper_2006_09791_amd import residual_block
    C = 256
    net = residual_block.random_blocks(C, 3, 0.2)
    x, dy = (torch.randn(4, 50, C, device="cuda").bfloat16() for _ in range(2))
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    tensors = lambda p: [p[0], p[1], p[3].dx, p[3].dpre_gamma] + [t for g, w in p[2] for t in (w, g.dh, g.dgate, g.dpost_gamma)]  # noqa: E731
    with on_side_stream(torch, b) as s:
        eager = net.train(x, dy, step)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = net.train(x, dy, step)
        for k in range(4):
            x.copy_(torch.randn_like(x))
            net.weights[k % 3].mul_(1.5)
            step.fill_(k)
            graph.replay()
            want = net.train(x, dy, step)
            s.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(tensors(held), tensors(want))), k
        del eager


def test_answers_are_of_the_weights_as_they_are(gpu):
    """Changed in place, by a write that torch does not see as one, or replaced: bit by bit a new network's answer, eager and replayed; rows that
    were laid out before are the caller's."""
    torch, b = gpu
    from paper_2006_09791_amd import residual_block
    C = 200
    net = residual_block.random_blocks(C, 2, seed=5)
    fresh = lambda: residual_block.ResidualBlocks(net.weights, net.gates, net.post, net.pre)  # noqa: E731
    x = torch.randn(2, 30, C, device="cuda").bfloat16()
    old, before = net.weight_rows(), net.answer(x)
    with on_side_stream(torch, b) as s:
        net.answer(x)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = net.answer(x)
        other = torch.randn(C, C, device="cuda") * 0.1
        for change in (lambda: net.weights[0].mul_(-1.5), lambda: net.weights[1].data.copy_(other), lambda: b.gspc_dropout(net.weights[0], 0.5, 3, out=net.weights[0])):
            last = net.answer(x)
            change()
            graph.replay()
            got, want = net.answer(x), fresh().answer(x)
            s.synchronize()
            assert torch.equal(got, want) and torch.equal(held, want) and not torch.equal(got, last)
        net.weights[0] = other
        got, want, given = net.answer(x), fresh().answer(x), net.answer(x, net.weight_rows())
        s.synchronize()
        assert torch.equal(got, want) and torch.equal(given, want)
        stale = net.answer(x, old)
        s.synchronize()
        assert torch.equal(stale, before)
    with pytest.raises(b.GspcError, match="rows of 1 weights"):
        net.answer(x, old[:1])


def test_command_prints_both_passes(gpu, capsys, monkeypatch):
    from paper_2006_09791_amd import residual_block
    monkeypatch.setattr("sys.argv", ["residual_block", "--images", "2", "--pixels", "5", "--channels", "72", "--blocks", "2", "--passes", "2"])
    residual_block.main()
    text = capsys.readouterr().out
    assert "answer:" in text and "train:" in text
