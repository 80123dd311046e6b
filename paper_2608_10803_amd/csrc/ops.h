// The operators of a transformer's feed-forward part beside the products:
// launch arguments shared by the C entry points (ops.cpp) and the kernels,
// and the library's error, workspace and launch-count services they use
// (adaptcore.cpp).
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <mutex>
#include <string>

#include "adaptcore.h"

namespace ac {

// ---- services of adaptcore.cpp
adaptcore_status op_fail(adaptcore_status st, const std::string& msg);  // records the thread's last error
adaptcore_status op_ready();                                             // device bound, gfx950
int op_compute_units();
adaptcore_hw_t op_hw();   // the planner's profile
void op_clear_choices();  // (ops.cpp) forgets what was chosen under it
// the library's workspace of (current device, stream), at least `bytes` long;
// keep `hold` until the call's last launch
adaptcore_status op_workspace(hipStream_t st, int64_t bytes, char** ptr, std::unique_lock<std::mutex>* hold);
void op_count_launches(int n);
// C = A B on the shape's cached plan (adaptcore_matmul, whatever override the
// thread holds), with the given workspace where ws is not null; and the most
// workspace a call of that plan takes
adaptcore_status op_matmul(int64_t M, int64_t N, int64_t K, int32_t dtype, uint32_t layouts, const void* A, int64_t lda,
                           const void* B, int64_t ldb, void* C, int64_t ldc, hipStream_t st, char* ws = nullptr,
                           int64_t ws_bytes = 0);
int64_t op_matmul_workspace(int64_t M, int64_t N, int64_t K, int32_t dtype, uint32_t layouts);

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

// ---- gated feed-forward block (kernels_ffn.hip). Operands are 16-byte
// aligned with pitches that are multiples of 8, at most DL_MAX_LD; LAY bits: 1: A
// stored as rows of M (k down the rows), 2: B stored as rows of K.
// One product of a launch: C (M x N) = A B over `K` then A2 B2 over another
// `K` (seg < blocks), in 64-deep k-blocks.
struct MultiProd {
  const uint16_t* A;
  const uint16_t* B;
  const uint16_t* A2;
  const uint16_t* B2;
  int64_t lda, ldb;
  int64_t M, N;
  int64_t eA, eB;  // rows of A and columns of B that may be loaded (along a stored row: rounded up to 8)
  int64_t kA, kB;  // k of a segment that may be loaded (along a stored row: rounded up to 8, zeros past K)
  void* C;
  int64_t ldc;
  float* part;  // pk slices of M x ldp partial sums (pk > 1)
  int64_t ldp;
  int tiles_m, tiles_n;
};
struct MultiArgs {
  MultiProd p[3];
  int n;
  int blocks;  // k-blocks of both segments
  int seg;     // first k-block of the second segment (blocks: none)
  int pk, kper;
};
// H (and, where G is not null, G and U) = both projections of X.
struct GatedArgs {
  const uint16_t* X;
  const uint16_t* Wg;
  const uint16_t* Wu;
  int64_t ldx, ldw;
  int64_t M, F;
  int64_t eF;      // features that may be loaded
  int64_t kX, kW;  // k that may be loaded (the loop runs over kX)
  uint16_t* H;
  int64_t ldh;
  uint16_t* H2;  // null, or H once more with zero-padded rows of whole aligned chunks
  int64_t ldh2;
  uint16_t* G;
  uint16_t* U;
  int64_t ldg;
  int act;
  int tiles_m, tiles_n;
};
// k_rows: C (M x N) = A B, B stored as N rows of K at any alignment; gated: B
// and B2 are both projections, C is H, and G and U (may be null) what they gave.
constexpr int64_t FFN_ROWS_MAX = 32;
struct RowsArgs {
  const uint16_t* A;
  const uint16_t* B;
  const uint16_t* B2;
  int64_t lda, ldb;
  int64_t M, N, K;
  void* C;
  int64_t ldc;
  uint16_t* G;
  uint16_t* U;
  int64_t ldg;
  int act;
};
// What k_dgate and k_dgate_sum do with dH (the product's M x N, N features):
// dG and dU (pitch ldd, 16-byte aligned, written up to N rounded up to 8).
struct DgateArgs {
  const uint16_t* G;
  const uint16_t* U;
  int64_t ldg;
  uint16_t* dG;
  uint16_t* dU;
  int64_t ldd;
  int act;
};
// Low-rank adapters (kernels_adapter.hip): n adapters, down n x R x K and up
// n x N x R with contiguous rows; T: M rows of ldt (R rounded up to 16) values,
// 16-byte aligned, of the input format for k_adapter, fp32 for k_adapter_sum.
struct AdapterArgs {
  const uint16_t* X;
  int64_t ldx;
  int64_t M, N, K;
  int n, R;
  const uint16_t* down;
  int64_t ld_down, stride_down;
  const uint16_t* up;
  int64_t ld_up, stride_up;
  const int32_t* index;
  const float* scale;  // null: 1
  const float* bias;   // null: none
  void* T;
  int64_t ldt;
  void* Y;
  int64_t ldy;
};
struct FfnTile {
  int bm, bn, stages;
};
// Zero-padded copies (k_pad_many): the caller fills the first row of fields.
struct PadMat {
  const uint16_t* src;
  uint16_t* dst;
  int64_t ld_src, ld_dst, rows, cols;
  int lg, per, blocks;
};
struct PadArgs {
  PadMat m[6];
  int n;
};
hipError_t launch_pad_many(PadArgs a, hipStream_t st);
#define AC_FFN_LAUNCHERS                                                                                          \
  hipError_t ffn_multi(const FfnTile& t, const MultiArgs& a, int lay, int out, hipStream_t st);                   \
  hipError_t ffn_dgate(const FfnTile& t, const MultiArgs& a, const DgateArgs& e, int lay, hipStream_t st);        \
  hipError_t ffn_gated(const FfnTile& t, const GatedArgs& g, int lay, hipStream_t st);                            \
  hipError_t ffn_rows(const RowsArgs& g, bool gated, hipStream_t st);                                             \
  hipError_t ffn_gated_sum(const MultiArgs& a, const GatedArgs& g, hipStream_t st);                               \
  hipError_t ffn_dgate_sum(const MultiArgs& a, const DgateArgs& e, hipStream_t st);                               \
  hipError_t ffn_plain_sum(const MultiArgs& a, int out, hipStream_t st);                                          \
  hipError_t adapter_shrink(const AdapterArgs& g, bool t16, hipStream_t st);                                      \
  hipError_t adapter_multi_shrink(const MultiArgs& a, const AdapterArgs& g, int lay, hipStream_t st);             \
  hipError_t adapter_tile(const FfnTile& t, const MultiArgs& a, const AdapterArgs& g, int lay, bool out16,        \
                          hipStream_t st);                                                                        \
  hipError_t adapter_sum(const MultiArgs& a, const AdapterArgs& g, bool out16, hipStream_t st);
AC_FFN_LAUNCHERS  // bf16; `out` 0: fp32, 1: the input format
namespace f16 {
AC_FFN_LAUNCHERS
}

}  // namespace ac
