"""ctypes binding of libadaptcore.so: argument marshalling only.

Every function has the name and argument order of the C entry point in
include/adaptcore.h. Device memory and streams are passed as integers
(addresses / hipStream_t handles); `torch` is optional and only used by the
convenience wrapper `matmul_tensors`. The library must be built
(`python -m paper_2608_10803_amd.build`); there is no fallback.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libadaptcore.so")

AC_N_CFG = 96  # calibrated cost table size (include/adaptcore.h)
AC_OK = 0
AC_ERR_INVALID_VALUE = -1
AC_ERR_UNSUPPORTED = -2
AC_ERR_OUT_OF_MEMORY = -3
AC_ERR_LAUNCH = -4
AC_ERR_NOT_INITIALIZED = -5
AC_ERR_INTERNAL = -6

AC_BF16_F32OUT = 0
AC_BF16_BF16OUT = 1
AC_F16_F32OUT = 2
AC_F16_F16OUT = 3
AC_FP16_F32OUT, AC_FP16_FP16OUT = AC_F16_F32OUT, AC_F16_F16OUT
AC_LAYOUT_ROW_ROW = 0
AC_LAYOUT_A_COL = 1  # A stored column-major (lda >= M)
AC_LAYOUT_B_COL = 2  # B stored column-major (ldb >= K)
AC_LAYOUT_COL_COL = 3
AC_A_ROWMAJOR, AC_A_COLMAJOR, AC_B_ROWMAJOR, AC_B_COLMAJOR = 0, AC_LAYOUT_A_COL, 0, AC_LAYOUT_B_COL
AC_TYPE_F32, AC_TYPE_BF16, AC_TYPE_F16 = range(3)  # element types of the operators beside the products
AC_ACT_SILU, AC_ACT_GELU, AC_ACT_GELU_TANH = range(3)
ACTIVATIONS = {"silu": AC_ACT_SILU, "gelu": AC_ACT_GELU, "gelu_tanh": AC_ACT_GELU_TANH}
AC_FFN_ROW, AC_FFN_UP_COL, AC_FFN_DOWN_COL = 0, 1, 2  # how the weights of a feed-forward block are stored
(AC_FAMILY_TILE, AC_FAMILY_SKINNY_M, AC_FAMILY_SKINNY_N, AC_FAMILY_STREAMK, AC_FAMILY_SMALLK, AC_FAMILY_DIRECT,
 AC_FAMILY_GROUPED, AC_FAMILY_PERSIST, AC_FAMILY_BATCHED, AC_FAMILY_DL, AC_FAMILY_TALL, AC_FAMILY_DL_OFFCHIP) = range(12)

CLASS_NAMES = ["Common", "SingleCoreSplitK", "MultiCoreSplitK", "HybridSplitK"]
FAMILY_NAMES = ["tile", "skinny_m", "skinny_n", "streamk", "smallk", "direct", "grouped", "persist", "batched", "dl",
                "tall", "offchip"]


class AdaptCoreError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("adaptcore error %d: %s" % (status, msg))
        self.status = status


class PlanDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("layouts", ctypes.c_uint32),
                ("shape_key", ctypes.c_uint64), ("variant_key", ctypes.c_uint64),
                ("cls", ctypes.c_int32), ("family", ctypes.c_int32),
                ("tile_m", ctypes.c_int32), ("tile_n", ctypes.c_int32), ("tile_k", ctypes.c_int32),
                ("pm", ctypes.c_int32), ("pn", ctypes.c_int32), ("pk", ctypes.c_int32),
                ("grid_x", ctypes.c_int32), ("grid_y", ctypes.c_int32),
                ("swizzle", ctypes.c_int32), ("n_candidates", ctypes.c_int32),
                ("predicted_s", ctypes.c_double), ("workspace_bytes", ctypes.c_int64),
                ("groups", ctypes.c_int64)]

    def as_dict(self):
        d = {f: getattr(self, f) for f, _ in self._fields_}
        d["cls_name"] = CLASS_NAMES[self.cls]
        d["family_name"] = FAMILY_NAMES[self.family]
        return d


class CallDesc(ctypes.Structure):
    _fields_ = [("variant_key", ctypes.c_uint64), ("in_place", ctypes.c_uint32), ("n_kernels", ctypes.c_int32),
                ("workspace_bytes", ctypes.c_int64), ("predicted_s", ctypes.c_double),
                ("kernels", ctypes.c_char * 256)]

    def as_dict(self):
        d = {f: getattr(self, f) for f, _ in self._fields_}
        d["kernels"] = [k for k in self.kernels.decode().split(";") if k]
        return d


class Candidate(ctypes.Structure):
    _fields_ = [("variant_key", ctypes.c_uint64), ("cls", ctypes.c_int32), ("family", ctypes.c_int32),
                ("tile_m", ctypes.c_int32), ("tile_n", ctypes.c_int32), ("tile_k", ctypes.c_int32),
                ("pk", ctypes.c_int32), ("grid_x", ctypes.c_int32), ("grid_y", ctypes.c_int32),
                ("predicted_s", ctypes.c_double)]

    def as_dict(self):
        d = {f: getattr(self, f) for f, _ in self._fields_}
        d["family_name"] = FAMILY_NAMES[self.family]
        return d


class Stats(ctypes.Structure):
    _fields_ = [("lookups", ctypes.c_uint64), ("hits", ctypes.c_uint64), ("misses", ctypes.c_uint64),
                ("entries", ctypes.c_uint64), ("launches", ctypes.c_uint64),
                ("miss_seconds", ctypes.c_double), ("class_count", ctypes.c_uint64 * 4)]


class Hw(ctypes.Structure):
    _fields_ = [("n_cu", ctypes.c_int32), ("lds_bytes", ctypes.c_int32), ("s_acc_bytes", ctypes.c_int64),
                ("clock_hz", ctypes.c_double), ("hbm_bw", ctypes.c_double), ("hbm_eta", ctypes.c_double),
                ("l2_bw_cu", ctypes.c_double), ("t_launch", ctypes.c_double),
                ("t_mem_latency", ctypes.c_double), ("t_wg", ctypes.c_double), ("mfma_eta", ctypes.c_double),
                ("lds_bw_cu", ctypes.c_double), ("unaligned_eta", ctypes.c_double), ("l2_hit", ctypes.c_double),
                ("search_open", ctypes.c_int32), ("enable_streamk", ctypes.c_int32),
                ("cfg_iter", ctypes.c_double * AC_N_CFG), ("cfg_wg", ctypes.c_double * AC_N_CFG),
                ("cfg_wr", ctypes.c_double * AC_N_CFG), ("swizzle_gain", ctypes.c_double)]

    def as_dict(self):
        d = {}
        for f, _ in self._fields_:
            v = getattr(self, f)
            d[f] = list(v) if f in ("cfg_iter", "cfg_wg", "cfg_wr") else v
        return d

    def copy(self):
        h = Hw()
        ctypes.memmove(ctypes.byref(h), ctypes.byref(self), ctypes.sizeof(Hw))
        return h


class TaxIn(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("M", "N", "K", "m", "n", "k", "m1", "n1", "k1", "n_core", "s_acc")] + \
               [("elem_bytes", ctypes.c_int32), ("out_bytes", ctypes.c_int32)]


class TaxOut(ctypes.Structure):
    _fields_ = [("pm", ctypes.c_int64), ("pn", ctypes.c_int64), ("pk", ctypes.c_int64), ("cls", ctypes.c_int32),
                ("acc_bytes", ctypes.c_int64), ("read_bytes", ctypes.c_double), ("write_bytes", ctypes.c_double)]


_lib = None


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libadaptcore.so is not built: run `python -m paper_2608_10803_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        i64, i32, u32, u64, p, d = (ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64,
                                    ctypes.c_void_p, ctypes.c_double)
        L.adaptcore_init.argtypes = []
        L.adaptcore_init.restype = i32
        L.adaptcore_plan.argtypes = [i64, i64, i64, i32, u32]
        L.adaptcore_plan.restype = p
        L.adaptcore_plan_variant.argtypes = [i64, i64, i64, i32, u32, u64]
        L.adaptcore_plan_variant.restype = p
        L.adaptcore_set_override.argtypes = [u64]
        L.adaptcore_set_override.restype = i32
        L.adaptcore_get_override.argtypes = []
        L.adaptcore_get_override.restype = u64
        L.adaptcore_matmul.argtypes = [p, p, i64, p, i64, p, i64, p]
        L.adaptcore_matmul.restype = i32
        L.adaptcore_matmul_shape.argtypes = [i64, i64, i64, i32, u32, p, i64, p, i64, p, i64, p]
        L.adaptcore_matmul_shape.restype = i32
        L.adaptcore_matmul_noalloc.argtypes = [p, p, i64, p, i64, p, i64, p]
        L.adaptcore_matmul_noalloc.restype = i32
        L.adaptcore_noalloc_scratch_bytes.argtypes = []
        L.adaptcore_noalloc_scratch_bytes.restype = i64
        L.adaptcore_addmm.argtypes = [p, p, i64, p, i64, p, i64, ctypes.c_float, ctypes.c_float, p, p]
        L.adaptcore_addmm.restype = i32
        L.adaptcore_grouped_plan.argtypes = [i64, i64, i64, i64, i32, u32]
        L.adaptcore_grouped_plan.restype = p
        L.adaptcore_grouped_plan_variant.argtypes = [i64, i64, i64, i64, i32, u32, u64]
        L.adaptcore_grouped_plan_variant.restype = p
        L.adaptcore_grouped_matmul.argtypes = [p, p, p, i64, p, i64, i64, p, i64, p]
        L.adaptcore_grouped_matmul.restype = i32
        L.adaptcore_batched_plan.argtypes = [i64, i64, i64, i64, i32, u32]
        L.adaptcore_batched_plan.restype = p
        L.adaptcore_batched_plan_variant.argtypes = [i64, i64, i64, i64, i32, u32, u64]
        L.adaptcore_batched_plan_variant.restype = p
        L.adaptcore_batched_matmul.argtypes = [p, p, i64, i64, p, i64, i64, p, i64, i64, p]
        L.adaptcore_batched_matmul.restype = i32
        L.adaptcore_batched_addmm.argtypes = [p, p, i64, i64, p, i64, i64, p, i64, i64, ctypes.c_float,
                                              ctypes.c_float, p, p]
        L.adaptcore_batched_addmm.restype = i32
        L.adaptcore_grouped_addmm.argtypes = [p, p, p, i64, p, i64, i64, p, i64, ctypes.c_float, ctypes.c_float, p,
                                              i64, p]
        L.adaptcore_grouped_addmm.restype = i32
        f32 = ctypes.c_float
        L.adaptcore_layer_norm.argtypes = [i64, i64, i32, i32, p, i64, p, p, f32, p, i64, p, p, p]
        L.adaptcore_layer_norm.restype = i32
        L.adaptcore_layer_norm_backward.argtypes = [i64, i64, i32, i32, p, i64, p, i64, p, p, p, p, i64, p, p, p]
        L.adaptcore_layer_norm_backward.restype = i32
        L.adaptcore_layer_norm_backward_workspace.argtypes = [i64, i64]
        L.adaptcore_layer_norm_backward_workspace.restype = i64
        L.adaptcore_gated_matmul.argtypes = [i64, i64, i64, i32, u32, i32, p, i64, p, p, i64, p, i64, p, p, i64, p]
        L.adaptcore_gated_matmul.restype = i32
        L.adaptcore_gated_ffn.argtypes = [i64, i64, i64, i32, u32, i32, p, i64, p, p, i64, p, i64, p, i64, p, p, i64, p,
                                          i64, p]
        L.adaptcore_gated_ffn.restype = i32
        L.adaptcore_gated_ffn_backward.argtypes = [i64, i64, i64, i32, u32, i32, p, i64, p, i64, p, p, i64, p, i64, p,
                                                   p, i64, p, i64, p, i64, i32, p, p, i64, p, i64, p]
        L.adaptcore_gated_ffn_backward.restype = i32
        L.adaptcore_gated_ffn_kernels.argtypes = [i64, i64, i64, u32, i32, ctypes.c_char_p, i64]
        L.adaptcore_gated_ffn_kernels.restype = i32
        L.adaptcore_gated_ffn_workspace.argtypes = [i64, i64, i64, i32]
        L.adaptcore_gated_ffn_workspace.restype = i64
        L.adaptcore_adapter_matmul.argtypes = [i64, i64, i64, i32, u32, p, i64, p, i64, i64, i64, p, i64, i64, p, i64,
                                               i64, p, p, p, p, i64, p]
        L.adaptcore_adapter_matmul.restype = i32
        L.adaptcore_adapter_workspace.argtypes = [i64, i64, i64, i64]
        L.adaptcore_adapter_workspace.restype = i64
        L.adaptcore_adapter_kernels.argtypes = [i64, i64, i64, ctypes.c_char_p, i64]
        L.adaptcore_adapter_kernels.restype = i32
        L.adaptcore_adapter_call_kernels.argtypes = [i64, i64, i64, i64, i64, ctypes.c_char_p, i64]
        L.adaptcore_adapter_call_kernels.restype = i32
        L.adaptcore_reserve_workspace.argtypes = [p, i64]
        L.adaptcore_reserve_workspace.restype = i32
        L.adaptcore_plan_info.argtypes = [p, ctypes.POINTER(PlanDesc)]
        L.adaptcore_plan_info.restype = i32
        L.adaptcore_plan_kernels.argtypes = [p, ctypes.c_char_p, i64]
        L.adaptcore_plan_kernels.restype = i32
        L.adaptcore_call_info.argtypes = [p, p, i64, i64, p, i64, i64, ctypes.POINTER(CallDesc)]
        L.adaptcore_call_info.restype = i32
        L.adaptcore_candidates.argtypes = [i64, i64, i64, i32, u32, ctypes.POINTER(Candidate), i64]
        L.adaptcore_candidates.restype = i64
        L.adaptcore_get_hw.argtypes = [ctypes.POINTER(Hw)]
        L.adaptcore_get_hw.restype = i32
        L.adaptcore_set_hw.argtypes = [ctypes.POINTER(Hw)]
        L.adaptcore_set_hw.restype = i32
        L.adaptcore_stats.argtypes = [ctypes.POINTER(Stats)]
        L.adaptcore_stats.restype = i32
        L.adaptcore_cache_clear.argtypes = []
        L.adaptcore_cache_clear.restype = i32
        L.adaptcore_bench_lookup.argtypes = [i64, i64, ctypes.POINTER(d)]
        L.adaptcore_bench_lookup.restype = i32
        L.adaptcore_read_probe.argtypes = [p, i64, p, p]
        L.adaptcore_read_probe.restype = i32
        L.adaptcore_last_error.argtypes = []
        L.adaptcore_last_error.restype = ctypes.c_char_p
        L.adaptcore_last_status.argtypes = []
        L.adaptcore_last_status.restype = i32
        L.adaptcore_taxonomy.argtypes = [ctypes.POINTER(TaxIn), ctypes.POINTER(TaxOut)]
        L.adaptcore_taxonomy.restype = i32
        L.adaptcore_schedule.argtypes = [i32, i64, i64, d, d, d]
        L.adaptcore_schedule.restype = d
        L.adaptcore_config_index.argtypes = [i32, i32]
        L.adaptcore_config_index.restype = i32
        _lib = L
    return _lib


def adaptcore_last_error():
    return lib().adaptcore_last_error().decode()


last_error = adaptcore_last_error


def adaptcore_last_status():
    return lib().adaptcore_last_status()


def _check(status):
    if status != AC_OK:
        raise AdaptCoreError(status, last_error())
    return status


def adaptcore_init():
    return _check(lib().adaptcore_init())


def adaptcore_plan(M, N, K, dtype=AC_BF16_BF16OUT, layouts=AC_LAYOUT_ROW_ROW):
    """Cached plan handle (int) for the shape."""
    h = lib().adaptcore_plan(M, N, K, dtype, layouts)
    if not h:
        raise AdaptCoreError(adaptcore_last_status(), last_error())
    return h


def adaptcore_plan_variant(M, N, K, dtype, layouts, variant_key):
    h = lib().adaptcore_plan_variant(M, N, K, dtype, layouts, variant_key)
    if not h:
        raise AdaptCoreError(adaptcore_last_status(), last_error())
    return h


def adaptcore_set_override(variant_key_or_0):
    """Force the configuration of this thread's later adaptcore_plan calls (0 = none)."""
    return _check(lib().adaptcore_set_override(variant_key_or_0))


def adaptcore_get_override():
    return lib().adaptcore_get_override()


def adaptcore_matmul(plan, A, lda, B, ldb, C, ldc, stream=0):
    """C = A * B on `stream`; A, B, C are device addresses (ints)."""
    return _check(lib().adaptcore_matmul(plan, A, lda, B, ldb, C, ldc, stream))


def adaptcore_matmul_shape(M, N, K, dtype, layouts, A, lda, B, ldb, C, ldc, stream=0):
    """adaptcore_plan and adaptcore_matmul in one call."""
    return _check(lib().adaptcore_matmul_shape(M, N, K, dtype, layouts, A, lda, B, ldb, C, ldc, stream))


def adaptcore_matmul_noalloc(plan, A, lda, B, ldb, C, ldc, stream=0):
    """adaptcore_matmul with the library's fixed device scratch as workspace
    (allocates nothing)."""
    return _check(lib().adaptcore_matmul_noalloc(plan, A, lda, B, ldb, C, ldc, stream))


def adaptcore_noalloc_scratch_bytes():
    return lib().adaptcore_noalloc_scratch_bytes()


def adaptcore_addmm(plan, A, lda, B, ldb, C, ldc, alpha=1.0, beta=0.0, bias=0, stream=0):
    """C = alpha * A * B + beta * C + bias on `stream`; A, B, C, bias are
    device addresses (ints), bias = 0 for none."""
    return _check(lib().adaptcore_addmm(plan, A, lda, B, ldb, C, ldc, alpha, beta, bias, stream))


def adaptcore_grouped_plan(rows, groups, N, K, dtype=AC_BF16_BF16OUT, layouts=AC_LAYOUT_ROW_ROW):
    """Cached grouped-product plan handle (int)."""
    h = lib().adaptcore_grouped_plan(rows, groups, N, K, dtype, layouts)
    if not h:
        raise AdaptCoreError(adaptcore_last_status(), last_error())
    return h


def adaptcore_grouped_plan_variant(rows, groups, N, K, dtype, layouts, variant_key):
    h = lib().adaptcore_grouped_plan_variant(rows, groups, N, K, dtype, layouts, variant_key)
    if not h:
        raise AdaptCoreError(adaptcore_last_status(), last_error())
    return h


def adaptcore_grouped_matmul(plan, counts, A, lda, B, ldb, stride_b, C, ldc, stream=0):
    """Grouped product on `stream`; counts, A, B, C are device addresses."""
    return _check(lib().adaptcore_grouped_matmul(plan, counts, A, lda, B, ldb, stride_b, C, ldc, stream))


def adaptcore_grouped_addmm(plan, counts, A, lda, B, ldb, stride_b, C, ldc, alpha=1.0, beta=0.0, bias=0,
                            stride_bias=0, stream=0):
    """Grouped product with the AddMM epilogue on `stream` (bias row of group
    g at bias + g * stride_bias floats; bias = 0 for none)."""
    return _check(lib().adaptcore_grouped_addmm(plan, counts, A, lda, B, ldb, stride_b, C, ldc, alpha, beta, bias,
                                                stride_bias, stream))


def adaptcore_batched_plan(batch, M, N, K, dtype=AC_BF16_BF16OUT, layouts=AC_LAYOUT_ROW_ROW):
    """Cached strided-batch plan handle (int)."""
    h = lib().adaptcore_batched_plan(batch, M, N, K, dtype, layouts)
    if not h:
        raise AdaptCoreError(adaptcore_last_status(), last_error())
    return h


def adaptcore_batched_plan_variant(batch, M, N, K, dtype, layouts, variant_key):
    h = lib().adaptcore_batched_plan_variant(batch, M, N, K, dtype, layouts, variant_key)
    if not h:
        raise AdaptCoreError(adaptcore_last_status(), last_error())
    return h


def adaptcore_batched_matmul(plan, A, lda, stride_a, B, ldb, stride_b, C, ldc, stride_c, stream=0):
    """Strided batched product on `stream`; A, B, C are device addresses."""
    return _check(lib().adaptcore_batched_matmul(plan, A, lda, stride_a, B, ldb, stride_b, C, ldc, stride_c, stream))


def adaptcore_batched_addmm(plan, A, lda, stride_a, B, ldb, stride_b, C, ldc, stride_c, alpha=1.0, beta=0.0, bias=0,
                            stream=0):
    """C_b = alpha * A_b B_b + beta * C_b + bias for every batch b on `stream`;
    A, B, C, bias are device addresses (bias = 0 for none)."""
    return _check(lib().adaptcore_batched_addmm(plan, A, lda, stride_a, B, ldb, stride_b, C, ldc, stride_c, alpha,
                                                beta, bias, stream))


def adaptcore_layer_norm(rows, cols, type, weight_type, X, ldx, weight, bias, eps, Y, ldy, mean=0, rstd=0, stream=0):
    """Layer norm of the rows of X on `stream`; addresses, 0 for an absent
    weight, bias, mean or rstd."""
    return _check(lib().adaptcore_layer_norm(rows, cols, type, weight_type, X, ldx, weight, bias, eps, Y, ldy, mean,
                                             rstd, stream))


def adaptcore_layer_norm_backward(rows, cols, type, weight_type, dY, lddy, X, ldx, weight, mean, rstd, dX, lddx,
                                  dweight=0, dbias=0, stream=0):
    """Backward pass of adaptcore_layer_norm on `stream`; addresses, 0 for an
    absent weight and for a weight gradient that is not wanted."""
    return _check(lib().adaptcore_layer_norm_backward(rows, cols, type, weight_type, dY, lddy, X, ldx, weight, mean,
                                                      rstd, dX, lddx, dweight, dbias, stream))


def adaptcore_layer_norm_backward_workspace(rows, cols):
    n = lib().adaptcore_layer_norm_backward_workspace(rows, cols)
    if n < 0:
        raise AdaptCoreError(n, last_error())
    return n


def adaptcore_gated_matmul(M, D, F, type, layouts, activation, X, ldx, Wg, Wu, ldw, H, ldh, G=0, U=0, ldg=1, stream=0):
    """H = act(X Wg) * (X Wu) on `stream`; addresses, G = U = 0 where the two
    products are not wanted."""
    return _check(lib().adaptcore_gated_matmul(M, D, F, type, layouts, activation, X, ldx, Wg, Wu, ldw, H, ldh, G, U,
                                               ldg, stream))


def adaptcore_gated_ffn(M, D, F, type, layouts, activation, X, ldx, Wg, Wu, ldw, Wd, ldd, H, ldh, G, U, ldg, Y, ldy,
                        stream=0):
    """adaptcore_gated_matmul, then Y = H Wd, on `stream`; addresses."""
    return _check(lib().adaptcore_gated_ffn(M, D, F, type, layouts, activation, X, ldx, Wg, Wu, ldw, Wd, ldd, H, ldh, G,
                                            U, ldg, Y, ldy, stream))


def adaptcore_gated_ffn_backward(M, D, F, type, layouts, activation, dY, lddy, X, ldx, Wg, Wu, ldw, Wd, ldd, G, U, ldg,
                                 H, ldh, dX, lddx, grad_type, dWg, dWu, lddw, dWd, lddd, stream=0):
    """Backward pass of adaptcore_gated_ffn on `stream`; addresses, 0 for
    gradients that are not wanted."""
    return _check(lib().adaptcore_gated_ffn_backward(M, D, F, type, layouts, activation, dY, lddy, X, ldx, Wg, Wu, ldw,
                                                     Wd, ldd, G, U, ldg, H, ldh, dX, lddx, grad_type, dWg, dWu, lddw,
                                                     dWd, lddd, stream))


def adaptcore_gated_ffn_workspace(M, D, F, backward=False):
    n = lib().adaptcore_gated_ffn_workspace(M, D, F, 1 if backward else 0)
    if n < 0:
        raise AdaptCoreError(n, last_error())
    return n


def adaptcore_gated_ffn_kernels(M, D, F, layouts=AC_FFN_ROW, backward=False):
    """What a call of these sizes launches, product by product."""
    buf = ctypes.create_string_buffer(256)
    _check(lib().adaptcore_gated_ffn_kernels(M, D, F, layouts, 1 if backward else 0, buf, len(buf)))
    return [k for k in buf.value.decode().split(";") if k]


def adaptcore_adapter_matmul(M, N, K, dtype, layouts, X, ldx, W, ldw, adapters, rank, down, ld_down, stride_down, up,
                             ld_up, stride_up, index, scale, bias, Y, ldy, stream=0):
    """Y = X W + bias with a low-rank adapter for each row, on `stream`;
    addresses, 0 for an absent scale or bias."""
    return _check(lib().adaptcore_adapter_matmul(M, N, K, dtype, layouts, X, ldx, W, ldw, adapters, rank, down, ld_down,
                                                 stride_down, up, ld_up, stride_up, index, scale, bias, Y, ldy, stream))


def adaptcore_adapter_workspace(M, N, K, rank):
    n = lib().adaptcore_adapter_workspace(M, N, K, rank)
    if n < 0:
        raise AdaptCoreError(n, last_error())
    return n


def adaptcore_adapter_kernels(M, N, K, rank=None, adapters=1):
    """What a call of these sizes on aligned operands launches. Without a rank:
    as with the highest, where the adapters' first product has a launch of its
    own."""
    if rank is not None:
        return adaptcore_adapter_call_kernels(M, N, K, adapters, rank)
    buf = ctypes.create_string_buffer(256)
    _check(lib().adaptcore_adapter_kernels(M, N, K, buf, len(buf)))
    return [k for k in buf.value.decode().split(";") if k]


def adaptcore_adapter_call_kernels(M, N, K, adapters, rank):
    """What a call with so many adapters of this rank launches."""
    buf = ctypes.create_string_buffer(256)
    _check(lib().adaptcore_adapter_call_kernels(M, N, K, adapters, rank, buf, len(buf)))
    return [k for k in buf.value.decode().split(";") if k]


def adaptcore_reserve_workspace(stream, nbytes):
    return _check(lib().adaptcore_reserve_workspace(stream, nbytes))


def adaptcore_plan_info(plan):
    d = PlanDesc()
    _check(lib().adaptcore_plan_info(plan, ctypes.byref(d)))
    return d.as_dict()


def adaptcore_plan_kernels(plan):
    """Kernels of the plan in launch order, in the form that operands of any
    alignment can take (what a call launches: adaptcore_call_info)."""
    buf = ctypes.create_string_buffer(512)
    _check(lib().adaptcore_plan_kernels(plan, buf, len(buf)))
    return buf.value.decode().split(";")


def adaptcore_call_info(plan, A, lda, B, ldb, stride_a=0, stride_b=0):
    """What one call of the plan on these operands launches (dict: variant_key,
    in_place, n_kernels, workspace_bytes, predicted_s, kernels)."""
    d = CallDesc()
    _check(lib().adaptcore_call_info(plan, A, lda, stride_a, B, ldb, stride_b, ctypes.byref(d)))
    return d.as_dict()


def adaptcore_candidates(M, N, K, dtype=AC_BF16_BF16OUT, layouts=AC_LAYOUT_ROW_ROW):
    n = lib().adaptcore_candidates(M, N, K, dtype, layouts, None, 0)
    if n < 0:
        raise AdaptCoreError(n, last_error())
    arr = (Candidate * max(n, 1))()
    lib().adaptcore_candidates(M, N, K, dtype, layouts, arr, n)
    return [arr[i].as_dict() for i in range(n)]


def adaptcore_get_hw():
    h = Hw()
    _check(lib().adaptcore_get_hw(ctypes.byref(h)))
    return h


def adaptcore_set_hw(h):
    return _check(lib().adaptcore_set_hw(ctypes.byref(h)))


def adaptcore_stats():
    s = Stats()
    _check(lib().adaptcore_stats(ctypes.byref(s)))
    d = {f: getattr(s, f) for f, _ in Stats._fields_ if f != "class_count"}
    d["class_count"] = list(s.class_count)
    return d


def adaptcore_cache_clear():
    return _check(lib().adaptcore_cache_clear())


def adaptcore_read_probe(buf, nbytes, sink, stream=0):
    """Measurement reference: read `nbytes` of the device buffer once."""
    return _check(lib().adaptcore_read_probe(buf, nbytes, sink, stream))


def adaptcore_bench_lookup(n_keys, n_lookups):
    out = ctypes.c_double()
    _check(lib().adaptcore_bench_lookup(n_keys, n_lookups, ctypes.byref(out)))
    return out.value


def adaptcore_taxonomy(M, N, K, m, n, k, m1, n1, k1, n_core, s_acc, elem_bytes=2, out_bytes=2):
    i = TaxIn(M, N, K, m, n, k, m1, n1, k1, n_core, s_acc, elem_bytes, out_bytes)
    o = TaxOut()
    _check(lib().adaptcore_taxonomy(ctypes.byref(i), ctypes.byref(o)))
    return {"pm": o.pm, "pn": o.pn, "pk": o.pk, "cls": CLASS_NAMES[o.cls], "acc_bytes": o.acc_bytes,
            "read_bytes": o.read_bytes, "write_bytes": o.write_bytes}


def adaptcore_config_index(family, cfg):
    return lib().adaptcore_config_index(family, cfg)


def adaptcore_schedule(kind, Q, L, t_m, t_p, t_drain):
    return lib().adaptcore_schedule(kind, Q, L, t_m, t_p, t_drain)


_torch = None       # the torch module, once a tensor wrapper has run
_dtype_codes = None  # (A, B, C torch dtypes) -> dtype code


def _bind_torch():
    global _torch, _dtype_codes
    import torch
    codes = {}
    for t, f32, same in ((torch.bfloat16, AC_BF16_F32OUT, AC_BF16_BF16OUT),
                         (torch.float16, AC_F16_F32OUT, AC_F16_F16OUT)):
        codes[t, t, torch.float32] = f32
        codes[t, t, t] = same
    _dtype_codes, _torch = codes, torch


def _current_stream():
    """Handle of the current device's current stream. (torch.cuda.
    current_stream() builds a Stream object around it, more than a microsecond
    of a call that takes eight in all.)"""
    c = _torch._C
    try:
        return c._cuda_getCurrentRawStream(c._cuda_getDevice())
    except AttributeError:
        return _torch.cuda.current_stream().cuda_stream


def _operand(t, rows, cols):
    """(column-major?, leading dimension) of a 2-D operand view: rows
    contiguous (stride(1) == 1) or columns contiguous (stride(0) == 1)."""
    if not t.is_cuda:
        raise ValueError("operands must be 2-D GPU tensors")
    sr, sc = t.stride()
    if cols <= 1 or sc == 1:
        col, ld, need = False, (sr if rows > 1 else cols), cols
    elif rows <= 1 or sr == 1:
        col, ld, need = True, (sc if cols > 1 else rows), rows
    else:
        raise ValueError("operands must have contiguous rows or contiguous columns")
    if ld < need:
        raise ValueError("overlapping operand view")
    return col, (ld if ld > 1 else 1)


def _marshal_tensors(A, B, C):
    """(M, N, K, dtype code, layouts, lda, ldb, ldc) of a tensor product,
    after the checks. A and B may be transposed views (contiguous columns);
    C must have contiguous rows."""
    if _torch is None:
        _bind_torch()
    M, K = A.shape
    K2, N = B.shape
    if K2 != K or C.shape != (M, N):
        raise ValueError("shape mismatch")
    dt = _dtype_codes.get((A.dtype, B.dtype, C.dtype))
    if dt is None:
        dt = _dtype_code(A, B, C)  # says what is wrong
    a_col, lda = _operand(A, M, K)
    b_col, ldb = _operand(B, K, N)
    sr, sc = C.stride()
    if not C.is_cuda or (N > 1 and sc != 1):
        raise ValueError("C must be a 2-D GPU tensor with contiguous rows")
    layouts = (AC_LAYOUT_A_COL if a_col else 0) | (AC_LAYOUT_B_COL if b_col else 0)
    return M, N, K, dt, layouts, lda, ldb, max(sr, N, 1)


def matmul_tensors(A, B, C, stream=None, plan=None):
    """C = A @ B for torch tensors on the GPU: 2-D, A and B with contiguous
    rows or contiguous columns (a transposed view selects the column-major
    layout), C with contiguous rows. A and B are both torch.bfloat16 or both
    torch.float16, C torch.float32 or the input type.
    Marshals pointers and leading dimensions; all arithmetic runs in the
    library's kernels."""
    M, N, K, dt, layouts, lda, ldb, ldc = _marshal_tensors(A, B, C)
    s = stream if stream is not None else _current_stream()
    if plan is None:
        _check((_lib or lib()).adaptcore_matmul_shape(M, N, K, dt, layouts, A.data_ptr(), lda, B.data_ptr(), ldb,
                                                      C.data_ptr(), ldc, s))
    else:
        adaptcore_matmul(plan, A.data_ptr(), lda, B.data_ptr(), ldb, C.data_ptr(), ldc, s)
    return C


def addmm_tensors(A, B, C, alpha=1.0, beta=0.0, bias=None, stream=None, plan=None):
    """C = alpha * A @ B + beta * C + bias in place, for torch tensors laid out
    as in matmul_tensors; bias is None or a contiguous float32 GPU tensor of
    N elements."""
    M, N, K, dt, layouts, lda, ldb, ldc = _marshal_tensors(A, B, C)
    bp = 0
    if bias is not None:
        if bias.dtype != _torch.float32 or bias.numel() != N or not bias.is_cuda or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous float32 GPU tensor of N elements")
        bp = bias.data_ptr()
    if plan is None:
        plan = adaptcore_plan(M, N, K, dt, layouts)
    s = stream if stream is not None else _current_stream()
    adaptcore_addmm(plan, A.data_ptr(), lda, B.data_ptr(), ldb, C.data_ptr(), ldc, float(alpha), float(beta), bp, s)
    return C


def _dtype_code(A, B, C):
    import torch
    if A.dtype != B.dtype or A.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("A and B must both be bfloat16 or both float16")
    f16 = A.dtype == torch.float16
    if C.dtype == torch.float32:
        return AC_F16_F32OUT if f16 else AC_BF16_F32OUT
    if C.dtype == A.dtype:
        return AC_F16_F16OUT if f16 else AC_BF16_BF16OUT
    raise TypeError("C must be float32 or the input type")


def _rows_contiguous(t, name):
    if not t.is_cuda or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError("%s must be a GPU tensor with contiguous rows" % name)


def bmm_tensors(A, B, C, alpha=None, beta=0.0, bias=None, stream=None, plan=None):
    """C[b] = A[b] @ B[b] for 3-D torch tensors on the GPU (batch x M x K,
    batch x K x N, batch x M x N; contiguous rows, any batch stride, B may be
    broadcast with batch stride 0). With alpha given: C[b] = alpha * A[b] @
    B[b] + beta * C[b] + bias (bias None or N float32 values), in place.
    Marshals pointers, leading dimensions and strides only."""
    if _torch is None:
        _bind_torch()
    batch, M, K = A.shape
    batch2, K2, N = B.shape
    if batch2 != batch or K2 != K or C.shape != (batch, M, N):
        raise ValueError("shape mismatch")
    dt = _dtype_codes.get((A.dtype, B.dtype, C.dtype))
    if dt is None:
        dt = _dtype_code(A, B, C)
    for t, n in ((A, "A"), (B, "B"), (C, "C")):
        _rows_contiguous(t, n)
    (sa, lda, _), (sb, ldb, _), (sc, ldc, _) = A.stride(), B.stride(), C.stride()
    lda, ldb, ldc = max(lda, K, 1), max(ldb, N, 1), max(ldc, N, 1)
    if plan is None:
        plan = adaptcore_batched_plan(batch, M, N, K, dt)
    s = stream if stream is not None else _current_stream()
    if alpha is None:
        adaptcore_batched_matmul(plan, A.data_ptr(), lda, sa, B.data_ptr(), ldb, sb, C.data_ptr(),
                                 ldc, sc, s)
    else:
        bp = 0
        if bias is not None:
            if bias.dtype != _torch.float32 or bias.numel() != N or not bias.is_cuda or not bias.is_contiguous():
                raise ValueError("bias must be a contiguous float32 GPU tensor of N elements")
            bp = bias.data_ptr()
        adaptcore_batched_addmm(plan, A.data_ptr(), lda, sa, B.data_ptr(), ldb, sb, C.data_ptr(),
                                ldc, sc, float(alpha), float(beta), bp, s)
    return C


def grouped_mm_tensors(A, B, counts, C, stream=None, plan=None):
    """The grouped product for torch tensors on the GPU: A (rows x K) holds
    the groups' rows one after another, B (groups x K x N, or K x N shared
    by all groups), counts an int32 GPU tensor of `groups` row counts (read by
    the kernel, never by the host), C (rows x N). Contiguous rows required.
    Marshals pointers, leading dimensions and strides only."""
    if _torch is None:
        _bind_torch()
    rows, K = A.shape
    if B.dim() == 2:
        groups, stride_b = counts.numel(), 0
        K2, N = B.shape
        ldb = max(B.stride(0), N, 1)
    else:
        groups, K2, N = B.shape
        stride_b, ldb = B.stride(0), max(B.stride(1), N, 1)
    if K2 != K or C.shape != (rows, N) or counts.numel() != groups:
        raise ValueError("shape mismatch")
    if counts.dtype != _torch.int32 or not counts.is_cuda or not counts.is_contiguous():
        raise ValueError("counts must be a contiguous int32 GPU tensor")
    dt = _dtype_codes.get((A.dtype, B.dtype, C.dtype))
    if dt is None:
        dt = _dtype_code(A, B, C)
    for t, n in ((A, "A"), (B, "B"), (C, "C")):
        _rows_contiguous(t, n)
    if plan is None:
        plan = adaptcore_grouped_plan(rows, groups, N, K, dt)
    s = stream if stream is not None else _current_stream()
    adaptcore_grouped_matmul(plan, counts.data_ptr(), A.data_ptr(), max(A.stride(0), K, 1), B.data_ptr(), ldb,
                             stride_b, C.data_ptr(), max(C.stride(0), N, 1), s)
    return C


_type_codes = None  # torch dtype -> adaptcore_type


def _type_of(t, name):
    global _type_codes
    if _type_codes is None:
        if _torch is None:
            _bind_torch()
        lib()
        _type_codes = {_torch.float32: AC_TYPE_F32, _torch.bfloat16: AC_TYPE_BF16, _torch.float16: AC_TYPE_F16}
    code = _type_codes.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float32, bfloat16 or float16" % name)
    return code


def _vector(t, n, dtype, name):
    """Address of a contiguous GPU vector of n elements (None: 0)."""
    if t is None:
        return 0
    if t.dtype is dtype and t.is_cuda and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    raise ValueError("%s must be a contiguous GPU tensor of %d elements" % (name, n))


def _rows_of(t, shape, dtype, name):
    """Row pitch of a 2-D GPU tensor of the given shape and type with
    contiguous rows that do not overlap (one row: its length, whatever its
    stride)."""
    if t.shape != shape:
        raise ValueError("%s: shape mismatch" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    rows, cols = shape
    sr, sc = t.stride()
    if t.is_cuda and sc == 1 and sr >= cols > 0:
        return sr if rows > 1 else cols
    if not t.is_cuda or (cols > 1 and sc != 1):
        raise ValueError("%s must be a GPU tensor with contiguous rows" % name)
    if rows > 1 and sr < cols:
        raise ValueError("%s: overlapping rows" % name)
    return max(sr if rows > 1 else cols, cols, 1)


def _norm_weights(X, *weights):
    """Type code and torch dtype of a norm's weights (float32 if there are
    none)."""
    for t in weights:
        if t is not None:
            return _type_of(t, "weights"), t.dtype
    return AC_TYPE_F32, _torch.float32


def layer_norm_tensors(X, weight, bias, Y, eps=1e-5, mean=None, rstd=None, stream=None):
    """Y = layer norm of the rows of X (2-D, contiguous rows of float32,
    bfloat16 or float16, any row pitch), into Y of the same shape and type.
    weight and bias: None, or `cols` values, both float32 or both of X's type;
    mean and rstd: None, or contiguous float32 tensors of `rows` values that
    receive the rows' statistics for the backward pass."""
    xt = _type_of(X, "X")
    shape, dtype = X.shape, X.dtype
    rows, cols = shape
    wt, wd = _norm_weights(X, weight, bias)
    f32 = _torch.float32
    status = _lib.adaptcore_layer_norm(
        rows, cols, xt, wt, X.data_ptr(), _rows_of(X, shape, dtype, "X"), _vector(weight, cols, wd, "weight"),
        _vector(bias, cols, wd, "bias"), eps, Y.data_ptr(), _rows_of(Y, shape, dtype, "Y"),
        _vector(mean, rows, f32, "mean"), _vector(rstd, rows, f32, "rstd"),
        _current_stream() if stream is None else stream)
    if status:
        _check(status)
    return Y


def layer_norm_backward_tensors(dY, X, weight, mean, rstd, dX, dweight=None, dbias=None, stream=None):
    """Backward pass of layer_norm_tensors: dX (of X's shape and type) and,
    where given, dweight and dbias (of the weight's type) from dY, X, weight
    (None: ones) and the rows' mean and rstd. dX may be dY or X itself."""
    xt = _type_of(X, "X")
    shape, dtype = X.shape, X.dtype
    rows, cols = shape
    wt, wd = _norm_weights(X, weight, dweight, dbias)
    f32 = _torch.float32
    if mean is None or rstd is None:
        raise ValueError("mean and rstd of the forward pass are needed")
    status = _lib.adaptcore_layer_norm_backward(
        rows, cols, xt, wt, dY.data_ptr(), _rows_of(dY, shape, dtype, "dY"), X.data_ptr(),
        _rows_of(X, shape, dtype, "X"), _vector(weight, cols, wd, "weight"), _vector(mean, rows, f32, "mean"),
        _vector(rstd, rows, f32, "rstd"), dX.data_ptr(), _rows_of(dX, shape, dtype, "dX"),
        _vector(dweight, cols, wd, "dweight"), _vector(dbias, cols, wd, "dbias"),
        _current_stream() if stream is None else stream)
    if status:
        _check(status)
    return dX


def _activation(name):
    code = ACTIVATIONS.get(name)
    if code is None:
        raise ValueError("act must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    return code


def _weight_of(t, shape, dtype, name):
    """(column-major?, pitch) of a weight of the given logical shape: rows
    contiguous, or a transposed view."""
    if t.shape != shape:
        raise ValueError("%s: shape mismatch" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    rows, cols = shape
    sr, sc = t.stride()
    if t.is_cuda and rows > 1 and cols > 1:
        if sr == 1 and sc >= rows:
            return True, sc
        if sc == 1 and sr >= cols:
            return False, sr
    return _operand(t, rows, cols)


def _weights_of(a, b, shape, dtype, names):
    """The same of two weights that lie alike."""
    la, lb = _weight_of(a, shape, dtype, names[0]), _weight_of(b, shape, dtype, names[1])
    if la != lb:
        raise ValueError("%s and %s must have the same layout and pitch" % names)
    return la


def _up_projections(X, Wg, Wu, H, gate, up):
    """The checked arguments that the block and its first half share."""
    xt = _type_of(X, "X")
    if xt == AC_TYPE_F32:
        raise TypeError("X must be bfloat16 or float16")
    shape, dtype = X.shape, X.dtype
    M, D = shape
    F = Wg.shape[1]
    col, ldw = _weights_of(Wg, Wu, (D, F), dtype, ("Wg", "Wu"))
    if (gate is None) != (up is None):
        raise ValueError("gate and up must both be given or both be None")
    gp = up_ = 0
    ldg = 1
    if gate is not None:
        ldg = _rows_of(gate, (M, F), dtype, "gate")
        if _rows_of(up, (M, F), dtype, "up") != ldg:
            raise ValueError("gate and up must have the same pitch")
        gp, up_ = gate.data_ptr(), up.data_ptr()
    return M, D, F, xt, col, _rows_of(X, shape, dtype, "X"), ldw, _rows_of(H, (M, F), dtype, "H"), gp, up_, ldg


def gated_mm_tensors(X, Wg, Wu, H, act="silu", gate=None, up=None, stream=None):
    """H = act(X @ Wg) * (X @ Wu) for 2-D bfloat16 or float16 GPU tensors: X
    (M x D) and H (M x F) with contiguous rows, Wg and Wu (D x F) alike, with
    contiguous rows or both transposed views (a linear layer's F x D weight).
    act: "silu", "gelu" or "gelu_tanh". gate and up (both or neither, alike)
    receive the two products, which the backward pass needs."""
    M, D, F, xt, col, ldx, ldw, ldh, gp, up_, ldg = _up_projections(X, Wg, Wu, H, gate, up)
    status = _lib.adaptcore_gated_matmul(
        M, D, F, xt, AC_FFN_UP_COL if col else 0, _activation(act), X.data_ptr(), ldx, Wg.data_ptr(), Wu.data_ptr(), ldw,
        H.data_ptr(), ldh, gp, up_, ldg, _current_stream() if stream is None else stream)
    if status:
        _check(status)
    return H


def gated_ffn_tensors(X, Wg, Wu, Wd, H, Y, act="silu", gate=None, up=None, stream=None):
    """The gated feed-forward block: gated_mm_tensors, then Y = H @ Wd. Wd
    (F x D) has contiguous rows or is a transposed view, Y (M x D) contiguous
    rows."""
    M, D, F, xt, col, ldx, ldw, ldh, gp, up_, ldg = _up_projections(X, Wg, Wu, H, gate, up)
    dcol, ldd = _weight_of(Wd, (F, D), X.dtype, "Wd")
    status = _lib.adaptcore_gated_ffn(
        M, D, F, xt, (AC_FFN_UP_COL if col else 0) | (AC_FFN_DOWN_COL if dcol else 0), _activation(act), X.data_ptr(), ldx,
        Wg.data_ptr(), Wu.data_ptr(), ldw, Wd.data_ptr(), ldd, H.data_ptr(), ldh, gp, up_, ldg, Y.data_ptr(),
        _rows_of(Y, X.shape, X.dtype, "Y"), _current_stream() if stream is None else stream)
    if status:
        _check(status)
    return Y


def gated_ffn_backward_tensors(dY, X, Wg, Wu, Wd, gate, up, H, dX=None, dWg=None, dWu=None, dWd=None, act="silu",
                               stream=None):
    """Backward pass of gated_ffn_tensors, from what it read and wrote (gate,
    up and H among it). Fills dX (X's shape and type), dWg and dWu (both or
    neither) and dWd where they are given; the weight gradients are laid out as
    their weights, all of X's type or all float32."""
    M, D, F, xt, col, ldx, ldw, ldh, gp, up_, ldg = _up_projections(X, Wg, Wu, H, gate, up)
    if gate is None:
        raise ValueError("gate and up of the forward pass are needed")
    dcol, ldd = _weight_of(Wd, (F, D), X.dtype, "Wd")
    lddy = _rows_of(dY, (M, D), X.dtype, "dY")
    lddx = _rows_of(dX, (M, D), X.dtype, "dX") if dX is not None else 1
    if (dWg is None) != (dWu is None):
        raise ValueError("dWg and dWu must both be given or both be None")
    some = dWg if dWg is not None else dWd
    gt, gd = (_type_of(some, "weight gradients"), some.dtype) if some is not None else (xt, X.dtype)
    lddw = lddd = 1
    if dWg is not None:
        gcol, lddw = _weights_of(dWg, dWu, (D, F), gd, ("dWg", "dWu"))
        if gcol != col:
            raise ValueError("dWg and dWu must be laid out as Wg and Wu")
    if dWd is not None:
        gcol, lddd = _weight_of(dWd, (F, D), gd, "dWd")
        if gcol != dcol:
            raise ValueError("dWd must be laid out as Wd")
    adaptcore_gated_ffn_backward(
        M, D, F, xt, (AC_FFN_UP_COL if col else 0) | (AC_FFN_DOWN_COL if dcol else 0), _activation(act), dY.data_ptr(),
        lddy, X.data_ptr(), ldx, Wg.data_ptr(), Wu.data_ptr(), ldw, Wd.data_ptr(), ldd, gp, up_, ldg, H.data_ptr(), ldh,
        dX.data_ptr() if dX is not None else 0, lddx, gt, dWg.data_ptr() if dWg is not None else 0,
        dWu.data_ptr() if dWu is not None else 0, lddw, dWd.data_ptr() if dWd is not None else 0, lddd,
        stream if stream is not None else _current_stream())
    return dX


def _stack(t, n, rows, cols, dtype, name):
    """(address, row pitch, stride) of n matrices with contiguous rows."""
    if t.shape != (n, rows, cols):
        raise ValueError("%s: shape mismatch" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    s0, s1, s2 = t.stride()
    if s2 == 1 and s1 >= cols > 0 and n > 1 and t.is_cuda:
        return t.data_ptr(), s1 if rows > 1 else cols, s0
    if not t.is_cuda or (cols > 1 and s2 != 1) or (rows > 1 and s1 < cols):
        raise ValueError("%s must be a GPU tensor with contiguous rows" % name)
    return t.data_ptr(), max(s1 if rows > 1 else cols, cols, 1), s0 if n > 1 else 0


def adapter_mm_tensors(X, W, down, up, index, Y, scale=None, bias=None, stream=None):
    """Y = X @ W + bias, and to every row i whose a = index[i] is one of the n
    adapters scale[a] * (X[i] @ down[a].T) @ up[a].T is added: low-rank adapters
    of many requests in one product. X (M x K) with contiguous rows, W (K x N)
    with contiguous rows or a transposed view, down (n x R x K) and up
    (n x N x R) with contiguous rows, all bfloat16 or all float16; index: int32
    (M), on the GPU, any order, -1 (or any other value outside) for rows without
    adapter; scale: None or n float32 values; bias: None or N; Y (M x N) of
    float32 or X's type with contiguous rows."""
    if _torch is None:
        _bind_torch()
    shape, dtype = X.shape, X.dtype
    M, K = shape
    N = W.shape[1]
    dt = _dtype_codes.get((dtype, W.dtype, Y.dtype))
    if dt is None:
        dt = _dtype_code(X, W, Y)
    if down.dim() != 3 or up.dim() != 3:
        raise ValueError("down and up must be stacks of matrices")
    n, R, _ = down.shape
    col, ldw = _weight_of(W, (K, N), dtype, "W")
    dp, ldd, sd = _stack(down, n, R, K, dtype, "down")
    pp, ldu, su = _stack(up, n, N, R, dtype, "up")
    f32 = _torch.float32
    status = (_lib or lib()).adaptcore_adapter_matmul(
        M, N, K, dt, AC_LAYOUT_B_COL if col else 0, X.data_ptr(), _rows_of(X, shape, dtype, "X"), W.data_ptr(), ldw, n, R,
        dp, ldd, sd, pp, ldu, su, _vector(index, M, _torch.int32, "index"), _vector(scale, n, f32, "scale"),
        _vector(bias, N, f32, "bias"), Y.data_ptr(), _rows_of(Y, (M, N), Y.dtype, "Y"),
        _current_stream() if stream is None else stream)
    if status:
        _check(status)
    return Y
