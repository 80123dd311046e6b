// The operators of a transformer's feed-forward part beside the products:
// launch arguments shared by the C entry points (ops.cpp) and the kernels,
// and the library's error, workspace and launch-count services they use
// (adaptcore.cpp).
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <string>

#include "adaptcore.h"

namespace ac {

// ---- services of adaptcore.cpp
adaptcore_status op_fail(adaptcore_status st, const std::string& msg);  // records the thread's last error
adaptcore_status op_ready();                                             // device bound, gfx950
int op_compute_units();
// the library's workspace of (current device, stream), at least `bytes` long
adaptcore_status op_workspace(hipStream_t st, int64_t bytes, char** ptr);
void op_count_launches(int n);

// ---- layer norm (kernels_norm.hip)
// Element types are adaptcore_type codes; the weights' is AC_TYPE_F32 or the
// rows'.
struct NormArgs {
  const void* x;
  int64_t ldx;
  const void* w;  // null: 1
  const void* b;  // null: 0
  void* y;
  int64_t ldy;
  float* mean;  // null: not written
  float* rstd;
  int64_t rows, cols;
  float eps;
};
struct NormBwdArgs {
  const void* dy;
  int64_t lddy;
  const void* x;
  int64_t ldx;
  const void* w;  // null: 1
  const float* mean;
  const float* rstd;
  void* dx;
  int64_t lddx;
  void* dw;  // null: not wanted
  void* db;
  int64_t rows, cols;
  float* part;  // partial weight gradients: `parts` rows of 2 * cols
  int parts;
};
hipError_t launch_norm(const NormArgs& a, int xt, int wt, int n_cu, hipStream_t st);
// partial rows of a backward call (0: neither weight gradient is wanted, or no rows)
int norm_bwd_parts(const NormBwdArgs& a, int n_cu);
hipError_t launch_norm_bwd(const NormBwdArgs& a, int xt, int wt, int n_cu, hipStream_t st, int* launches);

}  // namespace ac
