"""Parameterized fp32 GEMM and NHWC convolution forward for AMD MI355X (gfx950),
and the operators of a dense layer on 8-bit integers (``*_i8``).

The compute path is libpk.so (hand-written HIP kernels behind the C-ABI in
include/pk.h); this package only marshals arguments into it.
"""
from .binding import (PkError, PkLibraryMissing, configs, conv2d_fwd, conv2d_out_dims,  # noqa: F401
                      conv2d_same_pads, conv2d_winograd, conv2d_winograd_workspace_bytes,
                      conv2d_workspace_bytes, dequantize_i8, force_config, force_splits, gated_i8, gemm, gemm_i8,
                      quantize_i8, rmsnorm_i8, tune_conv2d, tune_gemm, tune_reset,
                      last_config_name, last_invalid_param, load)
