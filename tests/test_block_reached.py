"""Kernels of a residual block's operators without a GPU: calls reach each form that is compiled, and no other is."""
import itertools

import pytest

from paper_2006_09791_amd import binding as b
from test_block_launches import BASE, OUT, SC, ST, WS, launches
from test_block_resources import OPERATORS
from test_kernel_resources import kernels
from test_launches import runtime  # noqa: F401  (fixture)

ARGUMENTS = {name: [(-1, 0)] for name in OPERATORS}


def reached(runtime, calls):  # noqa: F811
    """Their kernels' whole names."""
    names = set()
    for (name, args), (rc, found) in zip(calls, launches(runtime, calls, ARGUMENTS)):
        assert rc == 0, (name, args)
        names |= {a[0].decode() for _, _, _, a in found}
    return names


def product(M, K, N, dtype):
    return "gspc_matmul_f8", [BASE, SC, OUT, ST, None, M, N, K, WS, dtype, N, WS, b.gspc_matmul_f8_workspace_bytes(M, N, K)]


PRODUCTS = [(1, 128, 16), (8, 4096, 4096), (200, 1024, 1024), (400, 1280, 1001), (1000, 2000, 3000), (2048, 512, 4096), (8192, 512, 4096), (1, 65536, 40),
            (300, 6400, 520), (256, 50176, 128)]


def residual(rows, C, gates, xt, ht, codes):
    """Forward and gradient."""
    post, pre, gates = (2, 1, gates) if ht is not None else (0, 1, 1)
    r = b.GspcResidual(rows, gates, C, post, pre, 0, None, None, None, None, ST if gates > 1 else None, 1.0, 1e-5, 0.0, 0, 0, None)
    h, raw = (BASE if ht is not None else None), list(bytes(r))
    z = [OUT, b.GSPC_F8, C, SC] if codes else [OUT, xt, C, None]
    need = b.gspc_residual_norm_backward_workspace_bytes(rows, C, gates)
    yield "gspc_residual_norm", [raw, BASE, xt, C, h, ht or 0, C, OUT, C, *z, ST]
    yield "gspc_residual_norm_backward", [raw, BASE, xt, C, BASE, C, BASE, xt, C, h, ht or 0, C, ST, OUT, C, OUT, C, None, None, None, ST, None, WS, need]


def rows(C, dtype):
    yield "gspc_quantize_rows_f8", [BASE, dtype, C, 40, C, OUT, SC, None, None]
    yield "gspc_quantize_rows_f8", [BASE, dtype, C, 40, C, OUT, SC, WS, ST]
    yield "gspc_dequantize_rows_f8", [OUT, SC, 40, C, BASE, dtype, C]
    yield "gspc_dropout", [BASE, dtype, C, 40, C, 0.5, 1, 2, None, OUT, C]


def test_every_kernel_is_reached(runtime):  # noqa: F811
    calls = [product(*s, t) for s in PRODUCTS for t in (0, 1)]
    calls += [c for C in (5, 60, 64) for t in (0, 1) for c in rows(C, t)]
    calls += [c for C, xt, ht, gates in itertools.product((5, 60, 64, 513, 1024, 8192), (0, 1), (None, 0, 1), (1, 40000))
              for c in residual(40000, C, gates, xt, ht, C == 64)]
    calls += list(residual(0, 64, 1, 0, None, False))
    names = reached(runtime, calls)
    compiled = {n for n in kernels() if any(f"{len(op)}{op}{end}" in n for op in OPERATORS for end in "IE")}
    assert compiled - names == set() and names <= compiled


@pytest.mark.parametrize("cols", [1, 31, 32, 33, 64, 200, 1000, 8192])
def test_parameters_sums_reach_every_column_once(runtime, cols):  # noqa: F811
    """A block of the join has 32 columns (kJoinCols), 1024 threads of them."""
    calls = list(residual(5000, cols, 4, 1, 1, False))[1:]
    (rc, found), = launches(runtime, calls, {"residual_join_kernel": [(4, 4)]})
    (blocks, threads, slabs), = [(n, threads, int.from_bytes(a[0], "little")) for k, n, threads, a in found if k == "residual_join_kernel"]
    assert rc == 0 and threads == 1024 and (slabs - 1) * 32 < cols <= slabs * 32 and blocks % slabs == 0


@pytest.mark.parametrize("M,K,N,waves", [(1000, 2000, 3000, 8), (2048, 512, 4096, 4)])
def test_tiles_of_128_in_four_and_eight_waves(runtime, M, K, N, waves):  # noqa: F811
    """Two forms that report one name: eight waves and four stages where a compute unit has one block."""
    for dtype in (0, 1):
        (rc, found), = launches(runtime, [product(M, K, N, dtype)], ARGUMENTS)
        (kernel, blocks, threads, (name,)), = found
        form = b"Li2ELi4ELi2ELi1ELi4E" if waves == 8 else b"Li2ELi2ELi2ELi2ELi2E"
        assert rc == 0 and kernel == "product_f8_tile_kernel" and form in name and threads == 64 * waves and blocks == -(-M // 128) * -(-N // 128)


@pytest.mark.parametrize("C,waves_of_a_team", [(264, 1), (320, 1), (512, 1), (520, 2), (640, 2), (1000, 2)])
def test_waves_of_the_gradient_go_by_tokens_of_a_team(runtime, C, waves_of_a_team):  # noqa: F811
    """Teams of one or two waves, four waves a block: twelve waves a compute unit from 8 tokens a team on, eight below, at any width."""
    full = 256 * 12 // waves_of_a_team          # teams
    for tokens, most in ((8 * full - 1, 8), (8 * full, 12), (11 * full + 77, 12), (40 * full, 12)):
        calls = list(residual(tokens, C, 1, 1, 1, False))[1:]
        (rc, found), = launches(runtime, calls, ARGUMENTS)
        (blocks, threads), = [(n, threads) for k, n, threads, _ in found if k == "residual_grad_kernel"]
        assert rc == 0 and threads == 256 and 0.9 * 256 * most < blocks * 4 <= 256 * most, (tokens, blocks)
