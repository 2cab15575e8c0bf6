"""Registers of the channels-last operators' kernels: none of them keeps values in scratch memory."""
from test_kernel_resources import kernels

OPERATORS = ("norm_stats_kernel", "norm_join_kernel", "norm_apply_kernel", "norm_rows_kernel", "norm_held_kernel", "norm_grad_sums_kernel",
             "norm_grad_join_kernel", "norm_grad_params_kernel", "norm_grad_apply_kernel", "norm_grad_held_kernel", "transpose_kernel",
             "transpose_thin_kernel", "quantize_rows_kernel", "dequantize_rows_kernel", "product8_small_kernel", "product8_tile_kernel")


def test_no_kernel_needs_scratch():
    found = dict.fromkeys(OPERATORS, 0)
    for n, k in kernels().items():
        for name in OPERATORS:
            if f"{len(name)}{name}I" in n or f"{len(name)}{name}E" in n:
                found[name] += 1
                assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
    assert all(found.values()), found
