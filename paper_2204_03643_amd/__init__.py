"""MI355X-native batched TV proximal operators (paper 2204.03643, Eq. 1-6, Alg. 1), and the channel products and
8-bit activation checkpoints of networks that hold them, with the borders of their residual blocks (norms, gate, scale,
dropout) and values and products in 4 bits for serving them.

A thin ctypes binding over the C-ABI library ``libtvprox.so`` (see ``include/tvprox.h``).
The modules are in ``layer`` (``TVLayer``), ``linear`` (``TVLinear``, ``TVMixer``), ``block`` (``TVNorm``,
``TVResidual``) and ``quant4`` (``TVLinear4``).
PyTorch is used only for device memory and streams; every step of the path runs in the
library's HIP kernels.  There is no CPU fallback: if the library is missing it is built
with hipcc, and if that fails the import raises.
"""
from .binding import (TVError, lib, status_str, tv_dispatch_thresholds, tv_dispatch_threshold, tv_dispatch_override, tv1d_bwd_workspace_bytes, tv1d_fwd_workspace_bytes,
                      tv1d_prox_fwd_ex, tv_fwd_extra, TV_FWD_ORDER_READY, TV_FWD_PARALLEL_SEARCH, tv1d_prox_fwd_steps,
                      tv1d_fwd_steps_floats_per_row, tv1d_prox_bwd, tv1d_prox_bwd_noalloc,
                      tv1d_prox_bwd_seg, tv1d_prox_fwd, tv1d_prox_fwd_info, tv1d_prox_fwd_seg, tv1d_prox_fwd_seg_bf16,
                      tv1d_prox_bwd_seg_bf16, tv2d_prox_bwd, tv2d_prox_fwd, tv2d_prox_fwd_bf16, tv2d_prox_bwd_bf16,
                      tv2d_workspace_bytes, tv_lambda, tv_rows, rows_along, tv_linear_desc, tv_held, tv_linear_fwd,
                      tv_linear_fwd_workspace_bytes, tv_linear_fwd_workspace_bytes_at, tv_linear_bwd,
                      tv_linear_bwd_workspace_bytes, tv_linear_bwd_workspace_bytes_at, tv_ckpt8_save,
                      tv_ckpt8_load, TV_F32, TV_BF16, TV_ACT_NONE, TV_ACT_RELU, TV_ACT_GELU, TV_ACT_SILU, TV_HELD_NONE,
                      TV_HELD_PLAIN, TV_HELD_BITS, TV_HELD_8BIT, TV_CKPT8_BLOCK,
                      tv_drop, tv_drop_apply, tv_block_desc, tv_block_in, tv_block_grads, tv_block_fwd,
                      tv_block_bwd, tv_block_bwd_workspace_bytes, tv_mx4_save, tv_mx4_load, tv_linear4_fwd,
                      tv_linear4_workspace_bytes, TV_NORM_NONE, TV_NORM_RMS, TV_NORM_LAYER, TV_GATE_PLAIN,
                      TV_GATE_SIGMOID, TV_GATE_SILU, TV_MAX_LENGTH, TV_MX4_GROUP)

__all__ = ["TVError", "lib", "status_str", "tv_dispatch_thresholds", "tv_dispatch_threshold", "tv_dispatch_override", "tv_rows", "tv_lambda", "rows_along", "tv1d_prox_fwd",
           "tv1d_prox_fwd_info", "tv1d_prox_bwd", "tv1d_prox_bwd_noalloc", "tv1d_prox_fwd_seg", "tv1d_prox_bwd_seg", "tv1d_prox_fwd_ex",
           "tv1d_prox_fwd_seg_bf16", "tv1d_prox_bwd_seg_bf16",
           "tv1d_fwd_workspace_bytes", "tv_fwd_extra", "TV_FWD_ORDER_READY", "TV_FWD_PARALLEL_SEARCH", "tv1d_prox_fwd_steps",
           "tv1d_fwd_steps_floats_per_row", "tv1d_bwd_workspace_bytes", "tv2d_prox_fwd",
           "tv2d_prox_bwd", "tv2d_workspace_bytes", "tv2d_prox_fwd_bf16", "tv2d_prox_bwd_bf16",
           "tv_linear_desc", "tv_held", "tv_linear_fwd", "tv_linear_fwd_workspace_bytes", "tv_linear_fwd_workspace_bytes_at", "tv_linear_bwd",
           "tv_linear_bwd_workspace_bytes", "tv_linear_bwd_workspace_bytes_at", "tv_ckpt8_save", "tv_ckpt8_load", "TV_F32", "TV_BF16", "TV_ACT_NONE",
           "TV_ACT_RELU", "TV_ACT_GELU", "TV_ACT_SILU", "TV_HELD_NONE", "TV_HELD_PLAIN", "TV_HELD_BITS", "TV_HELD_8BIT",
           "TV_CKPT8_BLOCK",
           "tv_drop", "tv_drop_apply", "tv_block_desc", "tv_block_in", "tv_block_grads", "tv_block_fwd", "tv_block_bwd",
           "tv_block_bwd_workspace_bytes", "tv_mx4_save", "tv_mx4_load", "tv_linear4_fwd", "tv_linear4_workspace_bytes",
           "TV_NORM_NONE", "TV_NORM_RMS", "TV_NORM_LAYER", "TV_GATE_PLAIN", "TV_GATE_SIGMOID", "TV_GATE_SILU",
           "TV_MAX_LENGTH", "TV_MX4_GROUP"]
