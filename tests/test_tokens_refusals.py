"""Channels-last operators: more refusals on the host, at the ends of what the arguments may be."""
import ctypes

from paper_2006_09791_amd import binding as b

P = ctypes.c_void_p(256 * 1024)                 # never dereferenced: validation fails first
DIM = -2


def test_norm_refuses_channels_whose_slabs_pass_32_bits():
    lib = b.load()
    for C in (0x7ffffff0, 0x7fffffff - 2046, 0x7fffffff - 4095):
        assert lib.gspc_group_norm_workspace_bytes(1, 1, C, 1, 0, 0) == 0 and "dimension" in b.gspc_last_error()
        assert lib.gspc_group_norm_backward_workspace_bytes(1, 1, C, 1, 0, 0) == 0
        assert lib.gspc_group_norm(P, 0, C, None, None, 1, 1, C, 1, 1e-5, 0, P, 0, C, None, None, None, None, P, 1 << 40) == DIM
        assert lib.gspc_group_norm_backward(P, 0, C, P, 0, C, None, P, None, None, 1, 1, C, 1, 0, P, C, P, P, P, 1 << 50) == DIM
    C = 0x7fffffff - 4096
    slabs = (C + 2047) // 2048
    assert lib.gspc_group_norm_workspace_bytes(1, 1, C, 1, 0, 0) == 8 + 8 * slabs
    assert lib.gspc_group_norm_backward_workspace_bytes(1, 1, C, 1, 0, 0) == (2 * C + 2 * C + 2) * 4
