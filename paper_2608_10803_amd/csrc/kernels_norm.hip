// gfx950 layer norm: y = (x - m) r w + b with the row's mean m and
// r = (v + eps)^-1/2, v the mean of (x - m)^2; and its backward pass
//   p = dy w, dx = r (p - mean(p) - xh mean(p xh)), xh = (x - m) r,
//   dw = sum over rows of dy xh, db = sum over rows of dy.
//
// Both are bound by HBM: a row is read once, held in registers as it came (16
// bytes for 8 elements), and written once. All sums are in fp32. The variance
// is the second pass over the held row, so a large mean costs no digits.
//
// A row belongs to WPR waves, VPT chunks of 8 elements a lane. Where the row's
// last chunk is not whole its lane takes the row's last 8 elements instead, and
// leaves those that are its neighbour's out of the sums (it writes them again,
// with the same values): every access is 16 bytes and no load waits for a
// branch. A workgroup
// walks rows with its columns' weights in registers (read once a workgroup
// instead of once a row: at 4096 columns of bf16 with fp32 weights they are
// four times the row itself) and the next row's loads issued before this row's
// reductions.
//
// The weight gradients: every lane keeps dw and db of its columns over the
// rows its workgroup walks, the workgroup writes them as one row of partial
// sums, and a second kernel adds the partial rows in a fixed order, so results
// do not depend on timing. (Atomics into dw would.)
//
// Measured, bf16 with fp32 weights: 8192 x 4096 forward 25 us (5.4 TB/s), backward
// 35 us (5.75 TB/s) and 4.7 us for the sum of 512 partial rows; a large device
// copy reaches 5.0. 16 x 4096 forward 4.3 us, 4099 x 1531 fp16 10 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops.h"

namespace ac {
namespace {

#include "row_ops.h"

// Rows in flight per workgroup: one with WPR > 1, a wave's each otherwise.
constexpr int norm_threads(int wpr) { return wpr == 1 ? 256 : 64 * wpr; }

template <int TX, int TW, int WPR, int VPT>
__global__ __launch_bounds__(norm_threads(WPR)) void k_norm(NormArgs a) {
  __shared__ float box[4 * WPR];
  int phase = 0;
  const int lane = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int cols = (int)a.cols;
  constexpr int RPB = WPR == 1 ? 4 : 1;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + (WPR == 1 ? threadIdx.x >> 6 : 0);
  const float inv = 1.0f / (float)a.cols;

  const auto span = [&](int v) { return Span((v * WPR * 64 + lane) * 8, cols); };
  Chunk<TX> next[VPT];
  if (r < a.rows) {
#pragma unroll
    for (int v = 0; v < VPT; ++v)
      next[v] = load_span<TX>(static_cast<const char*>(a.x) + r * a.ldx * elem_bytes(TX), span(v));
  }
  Chunk<TW> w[VPT], b[VPT];
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if (a.w) w[v] = load_span<TW>(a.w, span(v));
    if (a.b) b[v] = load_span<TW>(a.b, span(v));
  }
  // (with WPR > 1 the bound is the same for the whole workgroup, so every wave
  // meets every barrier)
  for (; r < a.rows; r += step) {
    float f[VPT][8], s = 0.f, none = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      unpack<TX>(next[v], f[v]);
      const int skip = span(v).skip;
#pragma unroll
      for (int e = 0; e < 8; ++e) s += e >= skip ? f[v][e] : 0.f;
    }
    if (r + step < a.rows) {
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        next[v] = load_span<TX>(static_cast<const char*>(a.x) + (r + step) * a.ldx * elem_bytes(TX), span(v));
    }
    row_sum2<WPR>(s, none, box, phase);
    const float mean = s * inv;
    float q = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int skip = span(v).skip;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[v][e] -= mean;
        q += e >= skip ? f[v][e] * f[v][e] : 0.f;
      }
    }
    row_sum2<WPR>(q, none, box, phase);
    const float rstd = 1.0f / sqrtf(q * inv + a.eps);
    if (lane == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      float wv[8], bv[8];
      unpack<TW>(w[v], wv);
      unpack<TW>(b[v], bv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float y = f[v][e] * rstd;
        if (a.w) y *= wv[e];
        if (a.b) y += bv[e];
        f[v][e] = y;
      }
      store_span<TX>(static_cast<char*>(a.y) + r * a.ldy * elem_bytes(TX), span(v), f[v]);
    }
  }
}

// Rows too long for registers, or of fewer than 8 elements: a workgroup of 16
// waves per row reads it three times (the second and third from the caches).
template <int TX, int TW>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a) {
  __shared__ float box[64];
  int phase = 0;
  const int cols = (int)a.cols;
  const float inv = 1.0f / (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const char* x = static_cast<const char*>(a.x) + r * a.ldx * elem_bytes(TX);
    float s = 0.f, none = 0.f;
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float f[8];
      unpack<TX>(load8<TX>(x, (int)c, cols), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += f[e];
    }
    row_sum2<16>(s, none, box, phase);
    const float mean = s * inv;
    float q = 0.f;
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float f[8];
      unpack<TX>(load8<TX>(x, (int)c, cols), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = c + e < cols ? f[e] - mean : 0.f;
        q += d * d;
      }
    }
    row_sum2<16>(q, none, box, phase);
    const float rstd = 1.0f / sqrtf(q * inv + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float f[8], wv[8], bv[8];
      unpack<TX>(load8<TX>(x, (int)c, cols), f);
      if (a.w) unpack<TW>(load8<TW>(a.w, (int)c, cols), wv);
      if (a.b) unpack<TW>(load8<TW>(a.b, (int)c, cols), bv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float y = (f[e] - mean) * rstd;
        if (a.w) y *= wv[e];
        if (a.b) y += bv[e];
        f[e] = y;
      }
      store8<TX>(static_cast<char*>(a.y) + r * a.ldy * elem_bytes(TX), (int)c, cols, f);
    }
  }
}

// ---- backward pass
// Rows in flight per workgroup: one with WPR > 1, eight otherwise (whose
// weight gradients are added in LDS at the end).
constexpr int bwd_threads(int wpr) { return wpr == 1 ? 512 : 64 * wpr; }

template <int TX, int TW, int WPR, int VPT>
__global__ __launch_bounds__(bwd_threads(WPR)) void k_norm_bwd(NormBwdArgs a) {
  __shared__ float box[4 * WPR];
  __shared__ float acc[WPR == 1 ? 8 * 512 : 1];
  int phase = 0;
  const int lane = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int cols = (int)a.cols;
  constexpr int RPB = WPR == 1 ? 8 : 1;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + (WPR == 1 ? threadIdx.x >> 6 : 0);
  const float inv = 1.0f / (float)a.cols;

  const auto span = [&](int v) { return Span((v * WPR * 64 + lane) * 8, cols); };
  Chunk<TX> nx[VPT], ny[VPT];
  float nm = 0.f, nr = 0.f;
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      nx[v] = load_span<TX>(static_cast<const char*>(a.x) + row * a.ldx * elem_bytes(TX), span(v));
      ny[v] = load_span<TX>(static_cast<const char*>(a.dy) + row * a.lddy * elem_bytes(TX), span(v));
    }
    nm = a.mean[row];
    nr = a.rstd[row];
  };
  if (r < a.rows) fetch(r);
  Chunk<TW> w[VPT];
  float dw[VPT][8], db[VPT][8];
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if (a.w) w[v] = load_span<TW>(a.w, span(v));
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[v][e] = db[v][e] = 0.f;
  }
  for (; r < a.rows; r += step) {
    float xh[VPT][8], p[VPT][8], s1 = 0.f, s2 = 0.f;
    const float mean = nm, rstd = nr;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      float g[8], wv[8];
      unpack<TX>(nx[v], xh[v]);
      unpack<TX>(ny[v], g);
      unpack<TW>(w[v], wv);
      const int skip = span(v).skip;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xh[v][e] = (xh[v][e] - mean) * rstd;
        dw[v][e] += g[e] * xh[v][e];
        db[v][e] += g[e];
        p[v][e] = a.w ? g[e] * wv[e] : g[e];
        s1 += e >= skip ? p[v][e] : 0.f;
        s2 += e >= skip ? p[v][e] * xh[v][e] : 0.f;
      }
    }
    if (r + step < a.rows) fetch(r + step);
    row_sum2<WPR>(s1, s2, box, phase);
    s1 *= inv;
    s2 *= inv;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[v][e] = rstd * (p[v][e] - s1 - xh[v][e] * s2);
      store_span<TX>(static_cast<char*>(a.dx) + r * a.lddx * elem_bytes(TX), span(v), p[v]);
    }
  }
  if (a.parts == 0) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const Span sp = span(v);
      if constexpr (WPR == 1) {
        // the eight waves' sums of 512 columns, added in their order (the last
        // chunk's where its columns are)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= sp.skip) acc[(threadIdx.x >> 6) * 512 + sp.at + e - v * 512] = k ? db[v][e] : dw[v][e];
        __syncthreads();
        const int col = v * 512 + threadIdx.x;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += acc[i * 512 + threadIdx.x];
        if (col < cols) part[(int64_t)k * cols + col] = s;
        __syncthreads();
      } else {
        // (another lane has the same sums of what this one skips)
        store_span<AC_TYPE_F32>(part + (k ? cols : 0), sp, k ? db[v] : dw[v]);
      }
    }
  }
}

// Such rows' dx with a workgroup of 16 waves per row, two
// passes over it.
template <int TX, int TW>
__global__ __launch_bounds__(1024) void k_norm_bwd_long(NormBwdArgs a) {
  __shared__ float box[64];
  int phase = 0;
  const int cols = (int)a.cols;
  const float inv = 1.0f / (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const char* x = static_cast<const char*>(a.x) + r * a.ldx * elem_bytes(TX);
    const char* dy = static_cast<const char*>(a.dy) + r * a.lddy * elem_bytes(TX);
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f;
    auto terms = [&](int c, float (&xh)[8], float (&p)[8]) {
      float wv[8];
      unpack<TX>(load8<TX>(x, c, cols), xh);
      unpack<TX>(load8<TX>(dy, c, cols), p);
      if (a.w) unpack<TW>(load8<TW>(a.w, c, cols), wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xh[e] = c + e < cols ? (xh[e] - mean) * rstd : 0.f;
        if (a.w) p[e] *= wv[e];
      }
    };
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float xh[8], p[8];
      terms((int)c, xh, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s1 += p[e];
        s2 += p[e] * xh[e];
      }
    }
    row_sum2<16>(s1, s2, box, phase);
    s1 *= inv;
    s2 *= inv;
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float xh[8], p[8];
      terms((int)c, xh, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = rstd * (p[e] - s1 - xh[e] * s2);
      store8<TX>(static_cast<char*>(a.dx) + r * a.lddx * elem_bytes(TX), (int)c, cols, p);
    }
  }
}

// The weight gradients of such rows: x: 2048 columns a workgroup, y: the rows
// in gridDim.y interleaved parts.
template <int TX>
__global__ __launch_bounds__(256) void k_norm_bwd_cols(NormBwdArgs a) {
  const int cols = (int)a.cols;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= cols) return;
  float dw[8] = {}, db[8] = {};
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    float x[8], g[8];
    unpack<TX>(load8<TX>(static_cast<const char*>(a.x) + r * a.ldx * elem_bytes(TX), (int)c, cols), x);
    unpack<TX>(load8<TX>(static_cast<const char*>(a.dy) + r * a.lddy * elem_bytes(TX), (int)c, cols), g);
    const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] += g[e] * ((x[e] - mean) * rstd);
      db[e] += g[e];
    }
  }
  float* part = a.part + (int64_t)blockIdx.y * 2 * cols;
  store8<AC_TYPE_F32>(part, (int)c, cols, dw);
  store8<AC_TYPE_F32>(part + cols, (int)c, cols, db);
}

// dw and db from the partial rows: a workgroup takes 32 columns of one of the
// two, 32 threads a column, added in a fixed order (512 partial rows of 4096
// columns: 5.0 us with 8 threads a column, one after the other's latency).
template <int TW>
__global__ __launch_bounds__(1024) void k_norm_bwd_sum(NormBwdArgs a) {
  __shared__ float s[1024];
  void* out = blockIdx.y ? a.db : a.dw;
  if (out == nullptr) return;
  const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  const int g = threadIdx.x >> 5;
  float v = 0.f;
  if (c < a.cols) {
    const float* p = a.part + (int64_t)blockIdx.y * a.cols + c;
#pragma unroll 8
    for (int i = g; i < a.parts; i += 32) v += p[(int64_t)i * 2 * a.cols];
  }
  s[threadIdx.x] = v;
  __syncthreads();
  if (g == 0 && c < a.cols) {
#pragma unroll
    for (int i = 1; i < 32; ++i) v += s[threadIdx.x + 32 * i];
    put<TW>(out, c, v);
  }
}

constexpr int MAX_BWD_COLS = 16384;

int64_t blocks_for(int64_t rows, int rows_per_block, int64_t most) {
  const int64_t n = (rows + rows_per_block - 1) / rows_per_block;
  return n < most ? n : most;
}

template <int TX, int TW, int WPR, int VPT>
void start_norm(const NormArgs& a, int n_cu, hipStream_t st) {
  // as many workgroups as the CUs hold at 2048 threads
  const int64_t n = blocks_for(a.rows, WPR == 1 ? 4 : 1, (int64_t)n_cu * (2048 / norm_threads(WPR)));
  hipLaunchKernelGGL((k_norm<TX, TW, WPR, VPT>), dim3((unsigned)n), dim3(norm_threads(WPR)), 0, st, a);
}
template <int TX, int TW>
void norm_typed(const NormArgs& a, int n_cu, hipStream_t st) {
  if (a.cols >= 8 && a.cols <= 512)
    start_norm<TX, TW, 1, 1>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 1024)
    start_norm<TX, TW, 1, 2>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 2048)
    start_norm<TX, TW, 4, 1>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 4096)
    start_norm<TX, TW, 4, 2>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 8192)
    start_norm<TX, TW, 8, 2>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 16384)
    start_norm<TX, TW, 16, 2>(a, n_cu, st);
  else
    hipLaunchKernelGGL((k_norm_long<TX, TW>), dim3((unsigned)blocks_for(a.rows, 1, (int64_t)n_cu * 2)), dim3(1024), 0,
                       st, a);
}

// workgroups of a backward call, each with one row of partial sums
int bwd_blocks(const NormBwdArgs& a, int n_cu) {
  if (a.cols <= 1024) return (int)blocks_for(a.rows, 8, 2 * n_cu);
  if (a.cols <= 4096) return (int)blocks_for(a.rows, 1, 2 * n_cu);
  return (int)blocks_for(a.rows, 1, n_cu);
}
template <int TX, int TW, int WPR, int VPT>
void start_bwd(const NormBwdArgs& a, int n_cu, hipStream_t st) {
  hipLaunchKernelGGL((k_norm_bwd<TX, TW, WPR, VPT>), dim3(bwd_blocks(a, n_cu)), dim3(bwd_threads(WPR)), 0, st, a);
}
// Rows of fewer than 8 elements, or too long for registers.
bool bwd_whole(const NormBwdArgs& a) { return a.cols >= 8 && a.cols <= MAX_BWD_COLS; }
template <int TX, int TW>
void bwd_long(const NormBwdArgs& a, int n_cu, hipStream_t st, int* n) {
  // the columns' sums first: dX may be written over dY or X
  if (a.parts > 0) {
    ++*n;
    hipLaunchKernelGGL((k_norm_bwd_cols<TX>), dim3((unsigned)((a.cols + 2047) / 2048), a.parts), dim3(256), 0, st, a);
  }
  hipLaunchKernelGGL((k_norm_bwd_long<TX, TW>), dim3((unsigned)blocks_for(a.rows, 1, (int64_t)n_cu * 2)), dim3(1024), 0,
                     st, a);
}
template <int TX, int TW>
int bwd_typed(const NormBwdArgs& a, int n_cu, hipStream_t st) {
  int n = 0;
  if (a.rows > 0) {
    ++n;
    if (!bwd_whole(a))
      bwd_long<TX, TW>(a, n_cu, st, &n);
    else if (a.cols <= 512)
      start_bwd<TX, TW, 1, 1>(a, n_cu, st);
    else if (a.cols <= 1024)
      start_bwd<TX, TW, 1, 2>(a, n_cu, st);
    else if (a.cols <= 2048)
      start_bwd<TX, TW, 4, 1>(a, n_cu, st);
    else if (a.cols <= 4096)
      start_bwd<TX, TW, 4, 2>(a, n_cu, st);
    else if (a.cols <= 8192)
      start_bwd<TX, TW, 8, 2>(a, n_cu, st);
    else
      start_bwd<TX, TW, 8, 4>(a, n_cu, st);
  }
  if (a.dw != nullptr || a.db != nullptr) {  // (no rows: zeros)
    ++n;
    hipLaunchKernelGGL((k_norm_bwd_sum<TW>), dim3((unsigned)((a.cols + 31) / 32), 2), dim3(1024), 0, st, a);
  }
  return n;
}

}  // namespace

int norm_bwd_parts(const NormBwdArgs& a, int n_cu) {
  if (a.rows <= 0 || (a.dw == nullptr && a.db == nullptr)) return 0;
  // long rows: a partial row costs as much as two rows of x, so few of them
  return bwd_whole(a) ? bwd_blocks(a, n_cu) : (int)(a.rows < 32 ? a.rows : 32);
}

hipError_t launch_norm(const NormArgs& a, int xt, int wt, int n_cu, hipStream_t st) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  if (xt == AC_TYPE_F32 && wt == AC_TYPE_F32)
    norm_typed<AC_TYPE_F32, AC_TYPE_F32>(a, n_cu, st);
  else if (xt == AC_TYPE_BF16 && wt == AC_TYPE_F32)
    norm_typed<AC_TYPE_BF16, AC_TYPE_F32>(a, n_cu, st);
  else if (xt == AC_TYPE_BF16 && wt == AC_TYPE_BF16)
    norm_typed<AC_TYPE_BF16, AC_TYPE_BF16>(a, n_cu, st);
  else if (xt == AC_TYPE_F16 && wt == AC_TYPE_F32)
    norm_typed<AC_TYPE_F16, AC_TYPE_F32>(a, n_cu, st);
  else if (xt == AC_TYPE_F16 && wt == AC_TYPE_F16)
    norm_typed<AC_TYPE_F16, AC_TYPE_F16>(a, n_cu, st);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormBwdArgs& a, int xt, int wt, int n_cu, hipStream_t st, int* launches) {
  *launches = 0;
  if (a.cols <= 0 || a.parts != norm_bwd_parts(a, n_cu) || (a.parts > 0 && a.part == nullptr))
    return a.cols <= 0 ? hipSuccess : hipErrorInvalidValue;
  if (xt == AC_TYPE_F32 && wt == AC_TYPE_F32)
    *launches = bwd_typed<AC_TYPE_F32, AC_TYPE_F32>(a, n_cu, st);
  else if (xt == AC_TYPE_BF16 && wt == AC_TYPE_F32)
    *launches = bwd_typed<AC_TYPE_BF16, AC_TYPE_F32>(a, n_cu, st);
  else if (xt == AC_TYPE_BF16 && wt == AC_TYPE_BF16)
    *launches = bwd_typed<AC_TYPE_BF16, AC_TYPE_BF16>(a, n_cu, st);
  else if (xt == AC_TYPE_F16 && wt == AC_TYPE_F32)
    *launches = bwd_typed<AC_TYPE_F16, AC_TYPE_F32>(a, n_cu, st);
  else if (xt == AC_TYPE_F16 && wt == AC_TYPE_F16)
    *launches = bwd_typed<AC_TYPE_F16, AC_TYPE_F16>(a, n_cu, st);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace ac
