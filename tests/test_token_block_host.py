"""The block's own tensors: made for the library's stream, whatever torch's current one is."""
import types

import pytest

from paper_2006_09791_amd import token_block

torch = pytest.importorskip("torch")


@pytest.fixture
def calls(monkeypatch):
    """(tensors made for the library's stream, arguments of the library's calls by name); nothing is computed."""
    made, seen, b = [], {}, token_block.b

    def empty(shape, dtype, device):
        made.append(torch.empty(shape, dtype=dtype, device=device))
        return made[-1]

    def stub(name, result):
        monkeypatch.setattr(b, name, lambda *a, **k: seen.update({name: (a, k)}) or result(a, k))
    monkeypatch.setattr(b, "_empty", empty)
    stub("gspc_conv2d_grouped", lambda a, k: k["output"] if k.get("output") is not None else a[12] if len(a) > 12 else torch.zeros(1))
    stub("gspc_output_dims", lambda a, k: (a[0], a[1]))
    stub("gspc_pack_channels_last", lambda a, k: "tokens")
    stub("gspc_group_norm", lambda a, k: "y")
    stub("gspc_group_norm_backward", lambda a, k: ("dx", "dgamma", "dbeta"))
    return made, seen


def block(C=32):
    t = object.__new__(token_block.TokenBlock)
    t.C, t.conv_groups, t.norm_groups, t.eps, t.packed, t.gamma, t.beta = C, 4, 8, 1e-5, types.SimpleNamespace(handle=None), None, None
    return t


def test_training_pass_keeps_tensors_of_the_librarys_stream(calls):
    made, seen = calls
    tokens = torch.zeros(2, 49, 32)
    assert block().train(tokens, tokens) == ("y", "dx", "dgamma", "dbeta")
    args = seen["gspc_group_norm"][1]
    kept = [args["stats"], *args["saved"]]
    assert [tuple(t.shape) for t in kept] == [(2, 8, 2), (98, 32), (98,)] and [t.dtype for t in kept] == [torch.float32, torch.int8, torch.float32]
    assert all(any(t is m for m in made) for t in kept)
    assert seen["gspc_group_norm_backward"][0][1:3] == (args["saved"], args["stats"])


def test_convolution_writes_a_tensor_of_the_librarys_stream(calls):
    made, seen = calls
    assert block().tokens(torch.zeros(2, 32, 7, 9)) == "tokens"
    y, = seen["gspc_pack_channels_last"][0]
    assert y.shape == (2, 32, 7, 9) and y.dtype == torch.float32 and any(y is m for m in made)
