"""How a residual block's operators are cut into launches: no launch has 2^32 threads or more, which the HIP runtime refuses, and the launches
of a call together reach every token once."""
import json
import subprocess
import sys

import pytest

import fake_runtime
from test_launches import number, runtime  # noqa: F401  (fixture)

b = fake_runtime.b
BASE, OUT, SC, ST, WS = (k << 44 for k in range(1, 6))         # addresses that nothing reads
CALLS = {"quantize_f8_kernel": [(0, 8), (2, 4), (6, 8), (7, 8)], "quantize_f8_turned_kernel": [(0, 8), (4, 4)],
         "dequantize_f8_kernel": [(0, 8), (1, 8), (2, 4), (6, 8)], "dropout_kernel": [(1, 8), (3, 4), (4, 4), (8, 8)]}


def launches(runtime, calls, decode):  # noqa: F811
    """As fake_runtime.launches, for calls whose first argument may be a description (its bytes), and with numbers in 64 bits."""
    child = fake_runtime.CHILD.replace("ctypes.c_float)}", "ctypes.c_float, ctypes.c_double)}").replace(
        "rc = call(*args)", "keep_r = (ctypes.c_char * len(args[0]))(*args[0]) if isinstance(args[0], list) else None\n"
        "    rc = call(ctypes.addressof(keep_r) if keep_r else args[0], *args[1:])")
    lib = b.load()
    kind = lambda t: getattr(t, "_type_", None) if isinstance(getattr(t, "_type_", None), str) else "P"  # noqa: E731  (a pointer to a description)
    work = [(name, [kind(t) for t in getattr(lib, name).argtypes], "i", args) for name, args in calls]
    out = subprocess.run([sys.executable, "-c", child, runtime, b.LIB_PATH], input=json.dumps({"calls": work, "decode": decode}), capture_output=True, text=True,
                         check=False, timeout=100)
    assert out.returncode == 0, out.stderr
    return [(rc, [(k, n, threads, [bytes.fromhex(v) for v in args]) for k, n, threads, args in found]) for rc, found in json.loads(out.stdout)]


@pytest.mark.parametrize("cols", [1, 128, 200, 4096])
@pytest.mark.parametrize("rows", [1, 1000, 0x7fffffff])
def test_rows_reach_every_row(runtime, rows, cols):  # noqa: F811
    pitch, s_pitch, blocks = b.gspc_f8_pitch(cols), b.gspc_f8_scale_pitch(cols), (cols + 127) // 128
    calls = [("gspc_quantize_rows_f8", [BASE, 1, cols, rows, cols, OUT, SC, None, None]), ("gspc_dequantize_rows_f8", [OUT, SC, rows, cols, BASE, 1, cols]),
             ("gspc_dropout", [BASE, 1, cols, rows, cols, 0.5, 1, 2, None, OUT, cols])]
    quantize, dequantize, dropout = launches(runtime, calls, CALLS)
    for rc, found in (quantize, dequantize, dropout):
        assert rc == 0 and all(blocks_ * threads < 1 << 32 for _, blocks_, threads, _ in found)
    at = 0
    for _, n, threads, (x, units, q, s) in quantize[1]:
        assert number(x) == BASE + 2 * at * cols and number(q) == OUT + at * pitch and number(s) == SC + at * s_pitch
        assert number(units) % blocks == 0 and n * threads // 16 >= number(units)
        at += number(units) // blocks
    assert at == rows
    at = 0
    for _, n, threads, (q, s, units, x) in dequantize[1]:
        assert number(x) == BASE + 2 * at * cols and number(q) == OUT + at * pitch and number(s) == SC + at * s_pitch
        at += number(units) // blocks
    assert at == rows
    at, nv = 0, (cols + 7) // 8
    for _, n, threads, (x, first, vectors, y) in dropout[1]:
        assert number(x) == BASE + 2 * at * cols and number(y) == OUT + 2 * at * cols and number(first) == at       # (rows keep their numbers)
        assert number(vectors) % nv == 0 and n * threads >= number(vectors)
        at += number(vectors) // nv
    assert at == rows


@pytest.mark.parametrize("rows,cols", [(1, 1), (129, 257), (0x7ffffc00, 100), (300, 0x7ffffc00)])
def test_turned_rows_reach_every_tile(runtime, rows, cols):  # noqa: F811
    (rc, found), = launches(runtime, [("gspc_quantize_rows_f8", [BASE, 0, cols, rows, cols, None, None, OUT, SC])], CALLS)
    assert rc == 0
    at = 0
    for _, n, threads, (x, first) in found:
        assert n * threads < 1 << 32 and number(x) == BASE and number(first) == at
        at += n
    assert at == (rows + 127) // 128 * ((cols + 127) // 128)


@pytest.mark.parametrize("M,K,N", [(1, 128, 1), (0x7fffffff, 100, 16), (100, 128, 0x7ffffff0), (70000, 256, 70000), (256, 50176, 128), (1, 65536, 64)])
def test_product_launches(runtime, M, K, N):  # noqa: F811
    need = b.gspc_matmul_f8_workspace_bytes(M, N, K)
    for dtype in (0, 1):
        (rc, found), = launches(runtime, [("gspc_matmul_f8", [BASE, SC, OUT, ST, None, M, N, K, WS, dtype, N, WS, need])], {})
        assert rc == 0 and found and all(n * threads < 1 << 32 for _, n, threads, _ in found)
    assert (need > 0) == (K > 10000)


@pytest.mark.parametrize("rows,cols,gates", [(1, 1, 1), (0x7fffffff, 8, 1), (0x7fffffff, 8, 0x7fffffff), (0x7fffffff, 8192, 1), (5365, 60, 5), (50176, 512, 1),
                                             (1 << 20, 8192, 1 << 20), (1 << 30, 512, 1 << 15)])
def test_residual_launches_reach_every_token(runtime, rows, cols, gates):  # noqa: F811
    r = b.GspcResidual(rows, gates, cols, 2, 1, 0, None, None, None, None, ST, 1.0, 1e-5, 0.0, 0, 0, None)
    raw = list(bytes(r))
    decode = {"residual_norm_kernel": [(2, 4), (3, 4)], "residual_grad_kernel": [(2, 16), (3, 4)], "residual_join_kernel": [(1, 4), (2, 4), (4, 4)]}
    need = b.gspc_residual_norm_backward_workspace_bytes(rows, cols, gates)
    forward = ("gspc_residual_norm", [raw, BASE, 1, cols, OUT, 1, cols, OUT, cols, OUT, 1, cols, None, ST])
    backward = ("gspc_residual_norm_backward", [raw, BASE, 1, cols, BASE, cols, BASE, 1, cols, OUT, 1, cols, ST, OUT, cols, OUT, cols, ST, ST, None, ST, None, WS, need])
    (rc, found), (rc2, grad) = launches(runtime, [forward, backward], decode)
    assert rc == rc2 == 0
    (_, n, threads, (team, each)), = found
    teams = threads // number(team)
    assert n * threads < 1 << 32 and (n - 1) * teams * number(each) < rows <= n * teams * number(each)
    assert number(team) * 8 >= cols and threads <= 1024
    (_, n, threads, (plan, team)) = grad[0]
    chunks, chunk_rows, each, blocks = (int.from_bytes(plan[4 * k:4 * k + 4], "little") for k in range(4))
    teams = threads // number(team)
    assert n == blocks and n * threads < 1 << 32 and need == n * 5 * cols * 4
    of_gate = rows // gates
    if chunks:                                  # blocks of one gate
        assert n == chunks * gates and (chunks - 1) * chunk_rows < of_gate <= chunks * chunk_rows <= chunks * teams * each and each <= 1024
    else:                                       # whole gates for each team
        assert each % of_gate == 0 and (n - 1) * teams * each < rows <= n * teams * each and each <= 1024       # (a sum's longest chain)
    (_, n, threads, (blocks, of, slabs)) = grad[1]
    assert number(blocks) == grad[0][1] and number(of) == chunks and n * threads < 1 << 32
    assert n == (4 + (gates if chunks > 1 else 0)) * number(slabs) and number(slabs) * 64 >= cols
