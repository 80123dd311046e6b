"""Adaptive dynamic-shape GEMM for MI355X (gfx950).

Python binding of the C ABI in include/adaptcore.h. The computation runs in
the HIP kernels of libadaptcore.so; this package only marshals arguments.
"""
from ._lib import *  # noqa: F401,F403
from ._lib import lib, last_error, AdaptCoreError, matmul_tensors, addmm_tensors, bmm_tensors, grouped_mm_tensors  # noqa: F401,E501
from ._lib import layer_norm_tensors, layer_norm_backward_tensors  # noqa: F401
from ._lib import gated_mm_tensors, gated_ffn_tensors, gated_ffn_backward_tensors, adapter_mm_tensors  # noqa: F401
