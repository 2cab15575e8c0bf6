"""MI355X (gfx950) library of grouped convolutions and of the channels-last operators between them: Python side.

`workloads` holds seeded input recipes; `binding` marshals arguments to the
C-ABI library libgspc.so, which does all the work in HIP kernels; `token_block`
is a network block made of both, `residual_block` a stack of residual blocks on tokens
(8-bit float products, norms with gate and residual, dropout), for answering and training.
"""
__all__ = ["workloads", "binding"]
