"""Registers of the residual block's kernels: none of them keeps values in scratch memory."""
from test_kernel_resources import kernels

OPERATORS = ("quantize_f8_kernel", "quantize_f8_turned_kernel", "dequantize_f8_kernel", "product_f8_small_kernel", "product_f8_tile_kernel",
             "product_f8_join_kernel", "dropout_kernel", "residual_norm_kernel", "residual_grad_kernel", "residual_join_kernel", "residual_clear_kernel")


def test_no_kernel_needs_scratch():
    found = dict.fromkeys(OPERATORS, 0)
    for n, k in kernels().items():
        for name in OPERATORS:
            if f"{len(name)}{name}I" in n or f"{len(name)}{name}E" in n:
                found[name] += 1
                assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
    assert all(found.values()), found
