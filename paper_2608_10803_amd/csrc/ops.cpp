// C entry points of the operators beside the products: checks, workspace,
// launches.
#include "ops.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace {

// No exception leaves a C entry point.
template <class F>
adaptcore_status guarded(F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return AC_ERR_OUT_OF_MEMORY;
  } catch (...) {
    return AC_ERR_INTERNAL;
  }
}

adaptcore_status launched(hipError_t e, int n) {
  if (e != hipSuccess)
    return ac::op_fail(AC_ERR_LAUNCH, std::string("kernel launch failed: ") + hipGetErrorString(e));
  ac::op_count_launches(n);
  return AC_OK;
}

adaptcore_status invalid(const char* msg) { return ac::op_fail(AC_ERR_INVALID_VALUE, msg); }
adaptcore_status unsupported(const char* msg) { return ac::op_fail(AC_ERR_UNSUPPORTED, msg); }

int type_bytes(int32_t t) { return t == AC_TYPE_F32 ? 4 : 2; }
bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// ---- layer norm
adaptcore_status norm_size(int64_t rows, int64_t cols) {
  if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 30))
    return invalid("rows must be in [0, 2^31) and cols in [0, 2^30)");
  return AC_OK;
}
adaptcore_status norm_types(int32_t type, int32_t weight_type) {
  if (type != AC_TYPE_F32 && type != AC_TYPE_BF16 && type != AC_TYPE_F16) return unsupported("unknown element type");
  if (weight_type != AC_TYPE_F32 && weight_type != type)
    return unsupported("the weights must be fp32 or of the rows' type");
  return AC_OK;
}

}  // namespace

extern "C" {

adaptcore_status adaptcore_layer_norm(int64_t rows, int64_t cols, int32_t type, int32_t weight_type, const void* X,
                                      int64_t ldx, const void* weight, const void* bias, float eps, void* Y,
                                      int64_t ldy, float* mean, float* rstd, void* stream) {
  return guarded([&] {
    adaptcore_status st = norm_size(rows, cols);
    if (st == AC_OK) st = norm_types(type, weight_type);
    if (st != AC_OK) return st;
    const int64_t need = std::max<int64_t>(1, cols);
    if (ldx < need || ldy < need) return invalid("row pitch smaller than the row");
    if (!std::isfinite(eps) || eps < 0) return invalid("eps must be finite and not negative");
    if (rows == 0 || cols == 0) return AC_OK;
    if (!X || !Y) return invalid("null matrix pointer");
    const int e = type_bytes(type), w = type_bytes(weight_type);
    if (misaligned(X, e) || misaligned(Y, e) || misaligned(weight, w) || misaligned(bias, w) || misaligned(mean, 4) ||
        misaligned(rstd, 4))
      return invalid("pointer not aligned to its element size");
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const ac::NormArgs a = {X, ldx, weight, bias, Y, ldy, mean, rstd, rows, cols, eps};
    return launched(
        ac::launch_norm(a, type, weight_type, ac::op_compute_units(), static_cast<hipStream_t>(stream)), 1);
  });
}

adaptcore_status adaptcore_layer_norm_backward(int64_t rows, int64_t cols, int32_t type, int32_t weight_type,
                                               const void* dY, int64_t lddy, const void* X, int64_t ldx,
                                               const void* weight, const float* mean, const float* rstd, void* dX,
                                               int64_t lddx, void* dweight, void* dbias, void* stream) {
  return guarded([&] {
    adaptcore_status st = norm_size(rows, cols);
    if (st == AC_OK) st = norm_types(type, weight_type);
    if (st != AC_OK) return st;
    const int64_t need = std::max<int64_t>(1, cols);
    if (lddy < need || ldx < need || lddx < need) return invalid("row pitch smaller than the row");
    if (cols == 0 || (rows == 0 && !dweight && !dbias)) return AC_OK;
    if (rows > 0 && (!dY || !X || !dX || !mean || !rstd)) return invalid("null pointer");
    const int e = type_bytes(type), w = type_bytes(weight_type);
    if (misaligned(dY, e) || misaligned(X, e) || misaligned(dX, e) || misaligned(weight, w) ||
        misaligned(dweight, w) || misaligned(dbias, w) || misaligned(mean, 4) || misaligned(rstd, 4))
      return invalid("pointer not aligned to its element size");
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const int n_cu = ac::op_compute_units();
    ac::NormBwdArgs a = {dY, lddy, X, ldx, weight, mean, rstd, dX, lddx, dweight, dbias, rows, cols, nullptr, 0};
    a.parts = ac::norm_bwd_parts(a, n_cu);
    if (a.parts > 0) {
      char* ws = nullptr;
      st = ac::op_workspace(static_cast<hipStream_t>(stream), (int64_t)a.parts * 2 * cols * 4, &ws);
      if (st != AC_OK) return st;
      a.part = reinterpret_cast<float*>(ws);
    }
    int n = 0;
    const hipError_t err =
        ac::launch_norm_bwd(a, type, weight_type, n_cu, static_cast<hipStream_t>(stream), &n);
    return launched(err, n);
  });
}

int64_t adaptcore_layer_norm_backward_workspace(int64_t rows, int64_t cols) {
  int64_t bytes = 0;
  const adaptcore_status st = guarded([&] {
    const adaptcore_status rc = norm_size(rows, cols);
    if (rc != AC_OK) return rc;
    ac::NormBwdArgs a;
    std::memset(&a, 0, sizeof a);
    a.rows = rows;
    a.cols = cols;
    a.dw = &bytes;  // any address: wanted
    if (cols > 0) bytes = (int64_t)ac::norm_bwd_parts(a, ac::op_compute_units()) * 2 * cols * 4;
    return AC_OK;
  });
  return st == AC_OK ? bytes : (int64_t)st;
}

}  // extern "C"
