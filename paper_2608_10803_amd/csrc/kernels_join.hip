// gfx950 kernels of the joint between a block and the residual stream, per row:
//   p = norm(y) w1 + b1 (or y),  r = s x + gate p,  n = norm(r) w2 + b2,
// norm(v) = (v - m) / sqrt(mean((v - m)^2) + eps) with m the mean (layer norm) or
// 0 (rms norm); and its backward pass, from dr, dn, x, y and the rows' statistics:
//   d  = dr + norm'(dn w2),   dx = s d,   dgate = sum d p,   dp = d gate,
//   dy = norm'(dp w1),  dw1 = sum dp xh1,  db1 = sum dp,  dw2 = sum dn xh2,  db2 = sum dn,
//   norm'(q) = rstd (q - mean(q) - xh mean(q xh)), without mean(q) for the rms norm.
//
// Bound by HBM: x and y are read once and r and n written once, where four
// operators of their own would move 9 matrices; the backward pass reads x, y, dr
// and dn and writes dx and dy. It computes r again from x and y, in the forward
// pass's 32 bits, instead of reading it rounded: as many bytes. 8192 x 4096 of bf16,
// rms norms and a gate: forward 52 us (268 MB, 5.1 TB/s), backward 87 (403 MB, 4.7
// TB/s) and 5 for the sums of the weights' gradients; N and its codes 64 (286 MB),
// codes alone 55 (219 MB), where N alone without statistics is 46. Sums by the
// registers' own exchanges and two rows on their way took the forward pass from 59, the
// same and the parts that a call does not have compiled out the backward pass from 112.
//
// Rows lie in registers as in kernels_norm.hip (row_ops.h): WPR waves a row, VPT
// chunks of eight elements a lane, the row's last chunk overlapping its
// neighbour, the next row's loads issued before this row's sums. (They are not long
// on their way alone: each load stands behind a condition, whether the lane has columns
// or the call that operand, so the compiler cannot count them and waits for all of a
// wave's loads and stores before it touches a row. Other workgroups of the CU hide that
// at 8192 x 4096; with two to five rows a workgroup nothing does.) Sums, statistics and
// gradients are fp32, added in an order that the sizes decide.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops.h"

#ifndef AC_JOIN_PART
#define AC_JOIN_PART 0
#endif

namespace ac {
namespace {

#include "row_ops.h"
#include "mx_format.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Sums over a wave in the registers' own paths (neighbours, mirrored halves and
// rows of 16 lanes, then the two exchanges of gfx950), where a shuffle through LDS
// costs a trip of 100 clocks a step.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_total(float v) {
  v += dpp<0xB1>(v);   // lanes 1 0 3 2
  v += dpp<0x4E>(v);   // lanes 2 3 0 1
  v += dpp<0x141>(v);  // halves of 16 lanes mirrored
  v += dpp<0x140>(v);  // 16 lanes mirrored
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Sums of N values over the WPR waves of a row; `box` and `phase` as row_sum2's, 2
// x WPR x N floats.
template <int WPR, int N>
__device__ __forceinline__ void row_total(float (&v)[N], float* box, int& phase) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_total(v[n]);
  if constexpr (WPR > 1) {
    float* half = box + phase * (N * WPR);
    phase ^= 1;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) half[N * w + n] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += half[N * i + n];
  }
}

// the row of a's gate that serves row r
__device__ __forceinline__ int64_t gate_row(const JoinArgs& a, int64_t r) {
  return (uint32_t)r / (uint32_t)a.per;  // (rows are below 2^31)
}

// the row's statistics (none are kept of a joint without norms: zeros)
__device__ __forceinline__ f32x4 row_stats(const JoinArgs& a, int64_t r) {
  f32x4 st = {};
  if (a.stats) __builtin_memcpy(&st, a.stats + 4 * r, 16);
  return st;
}

template <int T>
__device__ __forceinline__ const char* row_of(const void* p, int64_t ld, int64_t r) {
  return static_cast<const char*>(p) + r * ld * elem_bytes(T);
}
template <int T>
__device__ __forceinline__ char* row_of(void* p, int64_t ld, int64_t r) {
  return static_cast<char*>(p) + r * ld * elem_bytes(T);
}

// What a lane holds of the weights of its columns.
template <int TW, int VPT>
struct JoinWeights {
  Chunk<TW> w1[VPT], b1[VPT], gate[VPT], w2[VPT], b2[VPT];
};

// Codes of eight values of a row from column c on (a chunk's own place: f starts
// at `at` = c - skip), a quad of lanes a block; all lanes of the quad must be here.
template <int T>
__device__ __forceinline__ void put_codes(const JoinArgs& a, int64_t row, int c, const Span& sp, const float (&n)[8]) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {  // as the row's type holds them
    f[e] = n[e];
    if constexpr (T == AC_TYPE_BF16) f[e] = (float)(__bf16)f[e];
    if constexpr (T == AC_TYPE_F16) f[e] = (float)(_Float16)f[e];
  }
#pragma unroll
  for (int step = 4; step >= 1; step >>= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (sp.skip & step) ? (e + step < 8 ? f[e + step] : 0.f) : f[e];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = sp.skip == 8 ? 0.f : f[e];
  const uint32_t s = mx_scale_byte(mx_top_quad(mx_top8(f))), codes = mx_codes8(f, s);
  const int64_t blocks = (a.cols + 31) / 32;
  if ((c >> 5) < blocks) {
    __builtin_memcpy(a.codes + row * a.ld_codes + (c >> 1), &codes, 4);
    if ((c & 31) == 0) a.scales[row * a.ld_scales + (c >> 5)] = (uint8_t)s;
  }
}

constexpr int join_threads(int wpr) { return wpr == 1 ? 256 : 64 * wpr; }

// TX: the residual stream's type, TB: the block's, TW: the weights', which stay in
// registers from row to row. D: rows loaded ahead. (Rows of more than 8192 columns,
// 16 waves a row and weights read again for every row, 1000 x 16384: 92 us; k_join_long
// 46.)
template <int TX, int TB, int TW, int WPR, int VPT, int D>
__global__ __launch_bounds__(join_threads(WPR)) void k_join(JoinArgs a) {
  __shared__ float box[2 * WPR];
  int phase = 0;
  const int lane = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int cols = (int)a.cols;
  constexpr int RPB = WPR == 1 ? 4 : 1;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + (WPR == 1 ? threadIdx.x >> 6 : 0);
  const float inv = 1.0f / (float)a.cols;
  const bool many = a.gate && a.per < a.rows;  // a gate of its own for some rows

  const auto span = [&](int v) { return Span((v * WPR * 64 + lane) * 8, cols); };
  struct Next {
    Chunk<TX> x[VPT];
    Chunk<TB> y[VPT];
  } next[D];
  JoinWeights<TW, VPT> w;
  auto fetch = [&](Next& to, int64_t row) {
    if (row >= a.rows) return;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      to.x[v] = load_span<TX>(row_of<TX>(a.x, a.ldx, row), span(v));
      if (a.y) to.y[v] = load_span<TB>(row_of<TB>(a.y, a.ldy, row), span(v));
    }
  };
#pragma unroll
  for (int d = 0; d < D; ++d) fetch(next[d], r + d * step);
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if (a.w1) w.w1[v] = load_span<TW>(a.w1, span(v));
    if (a.b1) w.b1[v] = load_span<TW>(a.b1, span(v));
    if (a.gate && !many) w.gate[v] = load_span<TW>(a.gate, span(v));
    if (a.w2) w.w2[v] = load_span<TW>(a.w2, span(v));
    if (a.b2) w.b2[v] = load_span<TW>(a.b2, span(v));
  }
  auto work = [&](Next& of) {
    float f[VPT][8], p[VPT][8];
    float m1 = 0.f, r1 = 0.f, m2 = 0.f, r2 = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      unpack<TX>(of.x[v], f[v]);
      if (a.y) unpack<TB>(of.y[v], p[v]);
      if (many) w.gate[v] = load_span<TW>(row_of<TW>(a.gate, a.ld_gate, gate_row(a, r)), span(v));
    }
    if constexpr (WPR > 1) {
      // R may lie over X, and no lane may write what its neighbour, in another wave, has
      // yet to read: where the row's barriers are those of Y's sums alone, X is held
      // before them too. (8192 x 4096 of bf16 without N 32.8 us, not held 32.3; held
      // behind a branch for that case 33.2, and with N 46.4 instead of 45.9.)
#pragma unroll
      for (int v = 0; v < VPT; ++v) asm volatile("" ::"v"(f[v][0]), "v"(f[v][4]));
    }
    fetch(of, r + D * step);
    // the mean (layer norm) and 1 / deviation of a held row, which becomes its
    // differences from the mean
    auto norm = [&](float (&t)[VPT][8], float& m, float& rs) {
      m = 0.f;
      if (a.layer) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          const int skip = span(v).skip;
#pragma unroll
          for (int e = 0; e < 8; ++e) s[0] += e >= skip ? t[v][e] : 0.f;
        }
        row_total<WPR>(s, box, phase);
        m = s[0] * inv;
      }
      float q[1] = {0.f};
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        const int skip = span(v).skip;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[v][e] -= m;
          const float d = e >= skip ? t[v][e] : 0.f;
          q[0] += d * d;
        }
      }
      row_total<WPR>(q, box, phase);
      rs = 1.0f / sqrtf(q[0] * inv + a.eps);
    };
    if (a.post) norm(p, m1, r1);
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      if (a.post) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] *= r1;
        if (a.w1) {
          float t[8];
          unpack<TW>(w.w1[v], t);
#pragma unroll
          for (int e = 0; e < 8; ++e) p[v][e] *= t[e];
        }
        if (a.b1) {
          float t[8];
          unpack<TW>(w.b1[v], t);
#pragma unroll
          for (int e = 0; e < 8; ++e) p[v][e] += t[e];
        }
      }
      if (a.gate) {
        float t[8];
        unpack<TW>(w.gate[v], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] *= t[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) f[v][e] = a.y ? a.scale * f[v][e] + p[v][e] : a.scale * f[v][e];
    }
    if (!a.pre && !a.post) {
      // the same without any norm (the sums of R's norm, below, see to it themselves)
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < VPT; ++v) s[0] += f[v][0] + f[v][4];
      asm volatile("" ::"v"(s[0]));  // (what it waits for is what counts)
      row_total<WPR>(s, box, phase);
    }
    // R leaves after a sum over the row, when all of it is read
    if (a.pre) {
#pragma unroll
      for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] = f[v][e];
      norm(p, m2, r2);
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const Span sp = span(v);
      if (a.r) store_span<TX>(row_of<TX>(a.r, a.ldr, r), sp, f[v]);
      if (!a.pre) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[v][e] *= r2;
      if (a.w2) {
        float t[8];
        unpack<TW>(w.w2[v], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] *= t[e];
      }
      if (a.b2) {
        float t[8];
        unpack<TW>(w.b2[v], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] += t[e];
      }
      if (a.n) store_span<TB>(row_of<TB>(a.n, a.ldn, r), sp, p[v]);
      if (a.codes) put_codes<TB>(a, r, (v * WPR * 64 + lane) * 8, sp, p[v]);
    }
    if (lane == 0 && a.stats) {
      const float st[4] = {m1, r1, m2, r2};
      __builtin_memcpy(a.stats + 4 * r, st, 16);
    }
  };
  // (with WPR > 1 the bound is the same for the whole workgroup)
  while (r < a.rows) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (r >= a.rows) break;
      work(next[d]);
      r += step;
    }
  }
}

// Rows too long for registers, or of fewer than 8 elements: a workgroup of 16
// waves per row goes over it once for every sum and once to write it (from the
// caches after the first). Nothing of a row is written before its last pass.
template <int TX, int TB, int TW>
struct JoinRow {
  const JoinArgs& a;
  int64_t r;
  int cols;
  // p and R of the chunk at c, from the row's first statistics (rows past the
  // end: zeros)
  __device__ __forceinline__ void at(int c, float m1, float r1, float (&p)[8], float (&f)[8]) const {
    unpack<TX>(load8<TX>(row_of<TX>(a.x, a.ldx, r), c, cols), f);
    if (!a.y) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = 0.f;
        f[e] *= a.scale;
      }
      return;
    }
    unpack<TB>(load8<TB>(row_of<TB>(a.y, a.ldy, r), c, cols), p);
    affine(c, m1, r1, p);
    float g[8];
    gate(c, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = a.scale * f[e] + p[e] * g[e];
  }
  // y -> p
  __device__ __forceinline__ void affine(int c, float m1, float r1, float (&p)[8]) const {
    if (!a.post) return;
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = (p[e] - m1) * r1;
    if (a.w1) {
      unpack<TW>(load8<TW>(a.w1, c, cols), t);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] *= t[e];
    }
    if (a.b1) {
      unpack<TW>(load8<TW>(a.b1, c, cols), t);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] += t[e];
    }
  }
  __device__ __forceinline__ void gate(int c, float (&g)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = 1.f;
    if (a.gate) unpack<TW>(load8<TW>(row_of<TW>(a.gate, a.ld_gate, gate_row(a, r)), c, cols), g);
  }
  // sums over the row of get(c, value)[0 .. 7], and of the second
  template <class F>
  __device__ __forceinline__ void sums(float& s, float& t, float* box, int& phase, F get) const {
    s = t = 0.f;
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float u[8] = {}, v[8] = {};
      get((int)c, u, v);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < cols) {
          s += u[e];
          t += v[e];
        }
    }
    row_sum2<16>(s, t, box, phase);
  }
  // the mean and 1 / deviation of what get(c, value) gives
  template <class F>
  __device__ __forceinline__ void stats(float& m, float& rs, float* box, int& phase, F get) const {
    float none;
    const float inv = 1.0f / (float)cols;
    m = 0.f;
    if (a.layer) {
      sums(m, none, box, phase, [&](int c, float (&u)[8], float (&)[8]) { get(c, u); });
      m *= inv;
    }
    sums(rs, none, box, phase, [&](int c, float (&u)[8], float (&)[8]) {
      get(c, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = (u[e] - m) * (u[e] - m);
    });
    rs = 1.0f / sqrtf(rs * inv + a.eps);
  }
};
template <int TX, int TB, int TW>
__global__ __launch_bounds__(1024) void k_join_long(JoinArgs a) {
  __shared__ float box[64];
  int phase = 0;
  const int cols = (int)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const JoinRow<TX, TB, TW> row = {a, r, cols};
    float m1 = 0.f, r1 = 0.f, m2 = 0.f, r2 = 0.f;
    if (a.post)
      row.stats(m1, r1, box, phase, [&](int c, float (&u)[8]) { unpack<TB>(load8<TB>(row_of<TB>(a.y, a.ldy, r), c, cols), u); });
    if (a.pre)
      row.stats(m2, r2, box, phase, [&](int c, float (&u)[8]) {
        float p[8];
        row.at(c, m1, r1, p, u);
      });
    // (up to the end of the last block, for the codes)
    for (int64_t c = threadIdx.x * 8; c < (a.cols + 31) / 32 * 32; c += 8192) {
      float p[8], f[8];
      row.at((int)c, m1, r1, p, f);
      if (a.r) store8<TX>(row_of<TX>(a.r, a.ldr, r), (int)c, cols, f);
      if (!a.pre) continue;
      float t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (f[e] - m2) * r2;
      if (a.w2) {
        unpack<TW>(load8<TW>(a.w2, (int)c, cols), t);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= t[e];
      }
      if (a.b2) {
        unpack<TW>(load8<TW>(a.b2, (int)c, cols), t);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += t[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = c + e < cols ? f[e] : 0.f;
      if (a.n) store8<TB>(row_of<TB>(a.n, a.ldn, r), (int)c, cols, f);
      if (a.codes) {
        Span whole(0, 8);
        put_codes<TB>(a, r, (int)c, whole, f);
      }
    }
    if (threadIdx.x == 0 && a.stats) {
      const float st[4] = {m1, r1, m2, r2};
      __builtin_memcpy(a.stats + 4 * r, st, 16);
    }
  }
}

// ---- backward pass
// The gradients of the weights: every lane keeps those of its columns over the
// rows its workgroup walks, the workgroup writes them as one row of partial sums,
// and k_join_bwd_sum adds the partial rows in their order. A workgroup's rows are
// consecutive: a part of one group of rows with a common gate, whose gradient is
// a partial sum like the others, or whole groups, whose gradients it writes itself.
struct Rows {
  int64_t beg, end;
};
__device__ __forceinline__ Rows rows_of(const JoinBwdArgs& b, int64_t wg) {
  if (b.chunks > 0) {  // parts of a group
    const int64_t g = wg / b.chunks, beg = g * b.group + (wg - g * b.chunks) * b.rows_per;
    return {beg, min(beg + b.rows_per, (g + 1) * b.group)};
  }
  return {wg * b.rows_per, min((wg + 1) * b.rows_per, b.j.rows)};  // whole groups
}

constexpr int join_bwd_threads(int wpr) { return wpr == 1 ? 512 : 64 * wpr; }
enum JoinGrad { G_W1, G_B1, G_W2, G_B2, G_GATE, G_COUNT };

// D: rows loaded ahead. (Two rows at a time, whose sums share their barriers: 8192 x
// 4096 105 us instead of 100.) Two chunks a lane (4097 to 8192 columns) do not fit the
// registers: 68 to 512 bytes a lane lie in scratch memory, read again in the row loop
// (4096 x 8192 97 us, 4.1 TB/s, against 87 of 8192 x 4096). BIAS false: no post_bias, and no gradient of a bias is
// wanted (their registers). FULL: Y, both norms, dR and dN are there.
template <int TX, int TB, int TW, int WPR, int VPT, int D, bool BIAS, bool FULL>
__global__ __launch_bounds__(join_bwd_threads(WPR), 2) void k_join_bwd(JoinBwdArgs b) {
  const JoinArgs& a = b.j;
  __shared__ float box[2 * WPR * 2];
  __shared__ float cross[WPR == 1 ? 8 * 512 : 1];
  int phase = 0;
  const int lane = WPR == 1 ? threadIdx.x & 63 : threadIdx.x, wv = threadIdx.x >> 6;
  const int cols = (int)a.cols;
  constexpr int RPB = WPR == 1 ? 8 : 1;
  const float inv = 1.0f / (float)a.cols;
  const auto span = [&](int v) { return Span((v * WPR * 64 + lane) * 8, cols); };
  // a gate of its own for some rows, or for every row (its gradient is no sum then)
  const bool many = a.gate && a.per < a.rows, each = a.gate && a.per == 1;
  const bool row_gates = b.grad[G_GATE] && each;
  const bool has_y = FULL || a.y, post = FULL || a.post, has_dr = FULL || b.dr, has_dn = FULL || b.dn;
  const Rows mine = rows_of(b, blockIdx.x);

  struct Next {
    Chunk<TX> x[VPT], dr[VPT];
    Chunk<TB> y[VPT], dn[VPT];
    f32x4 stats;
  } next[D];
  JoinWeights<TW, VPT> w;
  float acc[G_COUNT][VPT][8];
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if (a.w1) w.w1[v] = load_span<TW>(a.w1, span(v));
    if (BIAS && a.b1) w.b1[v] = load_span<TW>(a.b1, span(v));
    if (a.gate && !many) w.gate[v] = load_span<TW>(a.gate, span(v));
    if (a.w2) w.w2[v] = load_span<TW>(a.w2, span(v));
#pragma unroll
    for (int k = 0; k < G_COUNT; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[k][v][e] = 0.f;
  }
  // (a row that is not there is zeros: it adds nothing to any sum)
  auto fetch = [&](Next& to, int64_t row, int64_t stop) {
    if (row >= stop) {
      to = Next{};
      return;
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      to.x[v] = load_span<TX>(row_of<TX>(a.x, a.ldx, row), span(v));
      if (has_y) to.y[v] = load_span<TB>(row_of<TB>(a.y, a.ldy, row), span(v));
      if (has_dr) to.dr[v] = load_span<TX>(row_of<TX>(b.dr, b.lddr, row), span(v));
      if (has_dn) to.dn[v] = load_span<TB>(row_of<TB>(b.dn, b.lddn, row), span(v));
    }
    if (FULL || a.stats) __builtin_memcpy(&to.stats, a.stats + 4 * row, 16);
  };
  // one lane's sums of all waves (with WPR > 1: its own)
  auto each_column = [&](const float (&t)[VPT][8], auto put_row, auto put_span) {
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const Span sp = span(v);
      if constexpr (WPR == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= sp.skip) cross[wv * 512 + sp.at + e - v * 512] = t[v][e];
        __syncthreads();
        const int col = v * 512 + threadIdx.x;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += cross[i * 512 + threadIdx.x];
        if (col < cols) put_row(col, s);
        __syncthreads();
      } else {
        put_span(sp, t[v]);
      }
    }
  };
  // rows of one gate at a time, but where every row has its own
  for (int64_t first = mine.beg; first < mine.end;) {
    int64_t stop = mine.end;
    if (many && !each) {
      stop = min(stop, (gate_row(a, first) + 1) * a.per);
#pragma unroll
      for (int v = 0; v < VPT; ++v) w.gate[v] = load_span<TW>(row_of<TW>(a.gate, a.ld_gate, gate_row(a, first)), span(v));
    }
    const int64_t r0 = first + (WPR == 1 ? wv : 0);
#pragma unroll
    for (int i = 0; i < D; ++i) fetch(next[i], r0 + i * RPB, stop);
    int64_t r = r0;
    auto work = [&](Next& of) {
      float x1[VPT][8], p[VPT][8], x2[VPT][8], d[VPT][8], q[VPT][8], s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
      const float m1 = of.stats[0], r1 = of.stats[1], m2 = of.stats[2], r2 = of.stats[3];
      auto gate_of = [&](int v, float (&g)[8]) {
        if (each)
          unpack<TW>(load_span<TW>(row_of<TW>(a.gate, a.ld_gate, r), span(v)), g);
        else
          unpack<TW>(w.gate[v], g);
      };
      {
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          const int skip = span(v).skip;
          float c[8];
          unpack<TX>(of.x[v], x2[v]);
#pragma unroll
          for (int e = 0; e < 8; ++e) x2[v][e] *= a.scale;
          if (has_y) {
            unpack<TB>(of.y[v], x1[v]);
            if (post) {
#pragma unroll
              for (int e = 0; e < 8; ++e) x1[v][e] = (x1[v][e] - m1) * r1;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) p[v][e] = x1[v][e];
            if (a.w1) {
              unpack<TW>(w.w1[v], c);
#pragma unroll
              for (int e = 0; e < 8; ++e) p[v][e] *= c[e];
            }
            if (BIAS && a.b1) {
              unpack<TW>(w.b1[v], c);
#pragma unroll
              for (int e = 0; e < 8; ++e) p[v][e] += c[e];
            }
            if (a.gate) {
              gate_of(v, c);
#pragma unroll
              for (int e = 0; e < 8; ++e) x2[v][e] += p[v][e] * c[e];
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) x2[v][e] += p[v][e];
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) d[v][e] = 0.f;
          if (has_dr) unpack<TX>(of.dr[v], d[v]);
          if (has_dn) {
            unpack<TB>(of.dn[v], q[v]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x2[v][e] = (x2[v][e] - m2) * r2;
              acc[G_W2][v][e] += q[v][e] * x2[v][e];
              if constexpr (BIAS) acc[G_B2][v][e] += q[v][e];
            }
            if (a.w2) {
              unpack<TW>(w.w2[v], c);
#pragma unroll
              for (int e = 0; e < 8; ++e) q[v][e] *= c[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float m = e >= skip ? q[v][e] : 0.f;
              s[0] += m;
              s[1] += m * x2[v][e];
            }
          }
        }
      }
      fetch(of, r + D * RPB, stop);
      if (has_dn) row_total<WPR>(s, box, phase);
      {
        const float s1 = a.layer ? s[0] * inv : 0.f, s2 = s[1] * inv;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          const Span sp = span(v);
          float c[8];
          if (has_dn) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d[v][e] += r2 * (q[v][e] - s1 - x2[v][e] * s2);
          }
          if (b.dx) {
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = a.scale * d[v][e];
            store_span<TX>(row_of<TX>(b.dx, b.lddx, r), sp, c);
          }
          if (!has_y) continue;
          if (row_gates) {
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = d[v][e] * p[v][e];
            store_span<TW>(row_of<TW>(b.grad[G_GATE], b.ld_dgate, r), sp, c);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[G_GATE][v][e] += d[v][e] * p[v][e];
          }
          if (a.gate) {
            gate_of(v, c);
#pragma unroll
            for (int e = 0; e < 8; ++e) d[v][e] *= c[e];
          }
          if (post) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              acc[G_W1][v][e] += d[v][e] * x1[v][e];
              if constexpr (BIAS) acc[G_B1][v][e] += d[v][e];
            }
            if (a.w1) {
              unpack<TW>(w.w1[v], c);
#pragma unroll
              for (int e = 0; e < 8; ++e) d[v][e] *= c[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float m = e >= sp.skip ? d[v][e] : 0.f;
              t[0] += m;
              t[1] += m * x1[v][e];
            }
          }
        }
      }
      if (!has_y) return;
      if (post) row_total<WPR>(t, box, phase);
      {
        const float t1 = a.layer ? t[0] * inv : 0.f, t2 = t[1] * inv;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          if (post) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d[v][e] = r1 * (d[v][e] - t1 - x1[v][e] * t2);
          }
          if (b.dy) store_span<TB>(row_of<TB>(b.dy, b.lddy, r), span(v), d[v]);
        }
      }
    };
    while (r < stop) {
#pragma unroll
      for (int i = 0; i < D; ++i) {
        if (r >= stop) break;
        work(next[i]);
        r += RPB;
      }
    }
    if (b.chunks == 0 && b.grad[G_GATE] && !row_gates) {  // this group's, whole
      char* out = row_of<TW>(b.grad[G_GATE], b.ld_dgate, gate_row(a, first));
      each_column(acc[G_GATE], [&](int col, float v) { put<TW>(out, col, v); },
                  [&](const Span& sp, const float (&v)[8]) { store_span<TW>(out, sp, v); });
#pragma unroll
      for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[G_GATE][v][e] = 0.f;
    }
    first = stop;
  }
  float* part = b.part + (int64_t)blockIdx.x * b.sections * cols;
#pragma unroll
  for (int k = 0; k < G_COUNT; ++k) {
    if (b.section[k] < 0 || (!BIAS && (k == G_B1 || k == G_B2))) continue;
    float* out = part + (int64_t)b.section[k] * cols;
    each_column(acc[k], [&](int col, float v) { out[col] = v; },
                [&](const Span& sp, const float (&v)[8]) { store_span<AC_TYPE_F32>(out, sp, v); });
  }
}

// Such rows' dx and dy with a workgroup of 16 waves per row, and the two means of
// norm'(dn w2), which the columns' sums need again.
template <int TX, int TB, int TW>
__global__ __launch_bounds__(1024) void k_join_bwd_long(JoinBwdArgs b) {
  const JoinArgs& a = b.j;
  __shared__ float box[64];
  int phase = 0;
  const int cols = (int)a.cols;
  const float inv = 1.0f / (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const JoinRow<TX, TB, TW> row = {a, r, cols};
    const f32x4 st = row_stats(a, r);
    const float m1 = st[0], r1 = st[1], m2 = st[2], r2 = st[3];
    float s1 = 0.f, s2 = 0.f, t1 = 0.f, t2 = 0.f;
    // dn w2 and xh2
    auto second = [&](int c, float (&q)[8], float (&x2)[8]) {
      float p[8];
      row.at(c, m1, r1, p, x2);
      unpack<TB>(load8<TB>(row_of<TB>(b.dn, b.lddn, r), c, cols), q);
#pragma unroll
      for (int e = 0; e < 8; ++e) x2[e] = (x2[e] - m2) * r2;
      if (a.w2) {
        float t[8];
        unpack<TW>(load8<TW>(a.w2, c, cols), t);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] *= t[e];
      }
    };
    if (b.dn) {
      row.sums(s1, s2, box, phase, [&](int c, float (&u)[8], float (&v)[8]) {
        second(c, u, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= u[e];
      });
      s1 = a.layer ? s1 * inv : 0.f;
      s2 *= inv;
    }
    if (threadIdx.x == 0 && b.means) {
      b.means[2 * r] = s1;
      b.means[2 * r + 1] = s2;
    }
    auto total = [&](int c, float (&d)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = 0.f;
      if (b.dr) unpack<TX>(load8<TX>(row_of<TX>(b.dr, b.lddr, r), c, cols), d);
      if (b.dn) {
        float q[8], x2[8];
        second(c, q, x2);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] += r2 * (q[e] - s1 - x2[e] * s2);
      }
    };
    // dp w1 and xh1
    auto firstn = [&](int c, float (&d)[8], float (&x1)[8]) {
      float g[8];
      total(c, d);
      row.gate(c, g);
      unpack<TB>(load8<TB>(row_of<TB>(a.y, a.ldy, r), c, cols), x1);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        d[e] *= g[e];
        x1[e] = (x1[e] - m1) * r1;
      }
      if (a.post && a.w1) {
        unpack<TW>(load8<TW>(a.w1, c, cols), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] *= g[e];
      }
    };
    if (a.y && a.post) {
      row.sums(t1, t2, box, phase, [&](int c, float (&u)[8], float (&v)[8]) {
        firstn(c, u, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= u[e];
      });
      t1 = a.layer ? t1 * inv : 0.f;
      t2 *= inv;
    }
    for (int64_t c = threadIdx.x * 8; c < cols; c += 8192) {
      float d[8], x1[8];
      if (b.dx) {
        total((int)c, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] *= a.scale;
        store8<TX>(row_of<TX>(b.dx, b.lddx, r), (int)c, cols, d);
      }
      if (a.y && b.dy) {
        firstn((int)c, d, x1);
        if (a.post) {
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = r1 * (d[e] - t1 - x1[e] * t2);
        }
        store8<TB>(row_of<TB>(b.dy, b.lddy, r), (int)c, cols, d);
      }
    }
  }
}
// The gradients of such rows' weights: x: 2048 columns a workgroup, y: one of the
// partial rows of k_join_bwd.
template <int TX, int TB, int TW>
__global__ __launch_bounds__(256) void k_join_bwd_cols(JoinBwdArgs b) {
  const JoinArgs& a = b.j;
  const int cols = (int)a.cols;
  const int64_t c64 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c64 >= cols) return;
  const int c = (int)c64;
  float acc[G_COUNT][8];
#pragma unroll
  for (int k = 0; k < G_COUNT; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[k][e] = 0.f;
  const Rows mine = rows_of(b, blockIdx.y);
  for (int64_t r = mine.beg; r < mine.end; ++r) {
    const JoinRow<TX, TB, TW> row = {a, r, cols};
    const f32x4 st = row_stats(a, r);
    const float m1 = st[0], r1 = st[1], m2 = st[2], r2 = st[3];
    float p[8], x2[8], d[8], g[8];
    row.at(c, m1, r1, p, x2);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = 0.f;
    if (b.dr) unpack<TX>(load8<TX>(row_of<TX>(b.dr, b.lddr, r), c, cols), d);
    if (b.dn) {
      float q[8], t[8];
      const float s1 = b.means[2 * r], s2 = b.means[2 * r + 1];
      unpack<TB>(load8<TB>(row_of<TB>(b.dn, b.lddn, r), c, cols), q);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x2[e] = (x2[e] - m2) * r2;
        acc[G_W2][e] += q[e] * x2[e];
        acc[G_B2][e] += q[e];
      }
      if (a.w2) {
        unpack<TW>(load8<TW>(a.w2, c, cols), t);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] *= t[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] += r2 * (q[e] - s1 - x2[e] * s2);
    }
    if (a.y) {
      row.gate(c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[G_GATE][e] += d[e] * p[e];
        d[e] *= g[e];
      }
      if (a.post) {
        unpack<TB>(load8<TB>(row_of<TB>(a.y, a.ldy, r), c, cols), p);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          acc[G_W1][e] += d[e] * ((p[e] - m1) * r1);
          acc[G_B1][e] += d[e];
        }
      }
    }
    if (b.chunks == 0 && b.grad[G_GATE] && (uint32_t)(r + 1) % (uint32_t)a.per == 0) {  // the group ends
      store8<TW>(row_of<TW>(b.grad[G_GATE], b.ld_dgate, gate_row(a, r)), c, cols, acc[G_GATE]);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[G_GATE][e] = 0.f;
    }
  }
  float* part = b.part + (int64_t)blockIdx.y * b.sections * cols;
#pragma unroll
  for (int k = 0; k < G_COUNT; ++k)
    if (b.section[k] >= 0) store8<AC_TYPE_F32>(part + (int64_t)b.section[k] * cols, c, cols, acc[k]);
}

// The gradients from the partial rows: `lanes` threads a column, eight partial rows
// each where there are as many, for 1024 / lanes columns of one of the weights', or
// of one group of the gate's, whose partial rows are its own; added in a fixed order.
// (32 threads a column and a workgroup for each of the gate's groups: 22 groups of 11
// partial rows and 2304 columns 11.9 us.)
struct JoinSums {
  const float* part;
  int64_t cols;
  int parts, sections, weights;  // partial rows, of so many gradients each; the gate's is the last
  int chunks;                    // partial rows of a group
  int lanes[2], blocks[2];       // of the weights', of the gate's: threads a column, workgroups a gradient
  void* out[G_COUNT];
  int64_t ld_gate, total;  // (workgroups' work)
};
template <int TW>
__global__ __launch_bounds__(1024) __attribute__((amdgpu_waves_per_eu(8))) void k_join_bwd_sum(JoinSums b) {
  __shared__ float s[1024];
  const int64_t first_gate = (int64_t)b.weights * b.blocks[0];
  for (int64_t id = blockIdx.x; id < b.total; id += gridDim.x) {
    const bool gate = id >= first_gate;
    const int64_t block = id - (gate ? first_gate : 0);
    const int blocks = b.blocks[gate], which = (int)(block / blocks), section = gate ? b.weights : which;
    const int lanes = b.lanes[gate], columns = 1024 / lanes, g = (int)threadIdx.x / columns;
    const int64_t c = (block - (int64_t)which * blocks) * columns + ((int)threadIdx.x & (columns - 1));
    const int64_t ld = (int64_t)b.sections * b.cols, first = gate ? (int64_t)which * b.chunks : 0;
    const int n = ((gate ? b.chunks : b.parts) - g + lanes - 1) / lanes;  // of the thread
    const float* const p = b.part + section * b.cols + min(c, b.cols - 1) + (first + g) * ld;
    float v = 0.f;
    for (int i = 0; i < n; i += 8) {
      float t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) t[u] = p[(int64_t)(min(i + u, n - 1) * lanes) * ld];
      __builtin_amdgcn_sched_barrier(0);  // (all of them on their way)
#pragma unroll
      for (int u = 0; u < 8; ++u) v += i + u < n ? t[u] : 0.f;
    }
    s[threadIdx.x] = v;
    __syncthreads();
    if (g == 0 && c < b.cols) {
#pragma unroll 8
      for (int i = 1; i < lanes; ++i) v += s[threadIdx.x + columns * i];
      put<TW>(gate ? row_of<TW>(b.out[section], b.ld_gate, which) : static_cast<char*>(b.out[section]), c, v);
    }
    __syncthreads();
  }
}
int sum_lanes(int rows) {
  int n = 1;
  while (n < 32 && n * 8 < rows) n *= 2;
  return n;
}

// ---- launches
constexpr int MAX_JOIN_BWD_COLS = 8192;
bool bwd_whole(int64_t cols) { return cols >= 8 && cols <= MAX_JOIN_BWD_COLS; }

int64_t blocks_for(int64_t rows, int rows_per_block, int64_t most) {
  const int64_t n = (rows + rows_per_block - 1) / rows_per_block;
  return n < most ? n : most;
}
template <int TX, int TB, int TW, int WPR, int VPT, int D>
void start(const JoinArgs& a, int n_cu, hipStream_t st) {
  // as many workgroups as the CUs hold at 1024 threads (at 2048: 8192 x 4096, with the
  // backward pass, 149 us against 145)
  const int64_t n = blocks_for(a.rows, WPR == 1 ? 4 : 1, (int64_t)n_cu * (1024 / join_threads(WPR)));
  hipLaunchKernelGGL((k_join<TX, TB, TW, WPR, VPT, D>), dim3((unsigned)n), dim3(join_threads(WPR)), 0, st, a);
}
template <int TX, int TB, int TW>
void join_typed(const JoinArgs& a, int n_cu, hipStream_t st) {
  if (a.cols >= 8 && a.cols <= 512)
    start<TX, TB, TW, 1, 1, 2>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 1024)
    start<TX, TB, TW, 1, 2, 1>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 2048)
    start<TX, TB, TW, 4, 1, 2>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 4096)
    start<TX, TB, TW, 8, 1, 2>(a, n_cu, st);
  else if (a.cols >= 8 && a.cols <= 8192)
    start<TX, TB, TW, 8, 2, 1>(a, n_cu, st);
  else
    hipLaunchKernelGGL((k_join_long<TX, TB, TW>), dim3((unsigned)blocks_for(a.rows, 1, (int64_t)n_cu * 2)), dim3(1024),
                       0, st, a);
}
template <int TX, int TB, int TW, int WPR, int VPT, int D, bool BIAS, bool FULL>
void start_bwd_of(const JoinBwdArgs& b, hipStream_t st) {
  hipLaunchKernelGGL((k_join_bwd<TX, TB, TW, WPR, VPT, D, BIAS, FULL>), dim3((unsigned)b.parts), dim3(join_bwd_threads(WPR)), 0, st, b);
}
template <int TX, int TB, int TW, int WPR, int VPT, int D>
void start_bwd(const JoinBwdArgs& b, hipStream_t st) {
  const JoinArgs& a = b.j;
  if (!a.y || !a.post || !b.dr || !b.dn)
    start_bwd_of<TX, TB, TW, WPR, VPT, D, true, false>(b, st);
  else if (a.b1 || b.grad[G_B1] || b.grad[G_B2])
    start_bwd_of<TX, TB, TW, WPR, VPT, D, true, true>(b, st);
  else
    start_bwd_of<TX, TB, TW, WPR, VPT, D, false, true>(b, st);
}
template <int TX, int TB, int TW>
int bwd_typed(const JoinBwdArgs& b, int n_cu, hipStream_t st) {
  int n = 0;
  const JoinArgs& a = b.j;
  if (a.rows > 0) {
    ++n;
    if (!bwd_whole(a.cols)) {
      hipLaunchKernelGGL((k_join_bwd_long<TX, TB, TW>), dim3((unsigned)blocks_for(a.rows, 1, (int64_t)n_cu * 2)),
                         dim3(1024), 0, st, b);
      if (b.sections > 0 || b.grad[G_GATE]) {
        ++n;
        hipLaunchKernelGGL((k_join_bwd_cols<TX, TB, TW>), dim3((unsigned)((a.cols + 2047) / 2048), (unsigned)b.parts),
                           dim3(256), 0, st, b);
      }
    } else if (a.cols <= 512) {
      start_bwd<TX, TB, TW, 1, 1, 1>(b, st);
    } else if (a.cols <= 1024) {
      start_bwd<TX, TB, TW, 2, 1, 2>(b, st);
    } else if (a.cols <= 2048) {
      start_bwd<TX, TB, TW, 4, 1, 2>(b, st);
    } else if (a.cols <= 4096) {
      start_bwd<TX, TB, TW, 8, 1, 2>(b, st);
    } else {
      start_bwd<TX, TB, TW, 8, 2, 1>(b, st);
    }
  }
  if (b.sections > 0) {  // (no rows: zeros)
    ++n;
    const bool gate = b.section[G_GATE] >= 0;
    const int weights = b.sections - (gate ? 1 : 0);
    JoinSums s = {b.part, a.cols, b.parts, b.sections, weights, b.chunks, {sum_lanes(b.parts), sum_lanes(b.chunks)}, {}, {},
                  b.ld_dgate, 0};
    for (int k = 0; k < 2; ++k) s.blocks[k] = (int)((a.cols * s.lanes[k] + 1023) / 1024);
    for (int k = 0; k < G_COUNT; ++k)
      if (b.section[k] >= 0) s.out[b.section[k]] = b.grad[k];
    s.total = (int64_t)weights * s.blocks[0] + (gate ? b.gate_rows * s.blocks[1] : 0);
    hipLaunchKernelGGL((k_join_bwd_sum<TW>), dim3((unsigned)blocks_for(s.total, 1, 1 << 16)), dim3(1024), 0, st, s);
  }
  return n;
}

}  // namespace

// Three parts: one type of the block each.
#if AC_JOIN_PART == 0
constexpr int JOIN_TB = AC_TYPE_BF16;
#define JOIN_NAME(n) n##_bf16
#elif AC_JOIN_PART == 1
constexpr int JOIN_TB = AC_TYPE_F16;
#define JOIN_NAME(n) n##_f16
#else
constexpr int JOIN_TB = AC_TYPE_F32;
#define JOIN_NAME(n) n##_f32
#endif

void JOIN_NAME(join)(const JoinArgs& a, bool res32, bool w32, int n_cu, hipStream_t st) {
#if AC_JOIN_PART < 2
  if (!res32 && !w32) return join_typed<JOIN_TB, JOIN_TB, JOIN_TB>(a, n_cu, st);
  if (!res32) return join_typed<JOIN_TB, JOIN_TB, AC_TYPE_F32>(a, n_cu, st);
  if (!w32) return join_typed<AC_TYPE_F32, JOIN_TB, JOIN_TB>(a, n_cu, st);
#endif
  join_typed<AC_TYPE_F32, JOIN_TB, AC_TYPE_F32>(a, n_cu, st);
}
int JOIN_NAME(join_bwd)(const JoinBwdArgs& b, bool res32, bool w32, int n_cu, hipStream_t st) {
#if AC_JOIN_PART < 2
  if (!res32 && !w32) return bwd_typed<JOIN_TB, JOIN_TB, JOIN_TB>(b, n_cu, st);
  if (!res32) return bwd_typed<JOIN_TB, JOIN_TB, AC_TYPE_F32>(b, n_cu, st);
  if (!w32) return bwd_typed<AC_TYPE_F32, JOIN_TB, JOIN_TB>(b, n_cu, st);
#endif
  return bwd_typed<AC_TYPE_F32, JOIN_TB, AC_TYPE_F32>(b, n_cu, st);
}

#if AC_JOIN_PART == 0
void join_f16(const JoinArgs& a, bool res32, bool w32, int n_cu, hipStream_t st);
void join_f32(const JoinArgs& a, bool res32, bool w32, int n_cu, hipStream_t st);
int join_bwd_f16(const JoinBwdArgs& b, bool res32, bool w32, int n_cu, hipStream_t st);
int join_bwd_f32(const JoinBwdArgs& b, bool res32, bool w32, int n_cu, hipStream_t st);

hipError_t launch_join(const JoinArgs& a, int rt, int bt, int wt, int n_cu, hipStream_t st) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  const bool r32 = rt == AC_TYPE_F32, w32 = wt == AC_TYPE_F32;
  if (bt == AC_TYPE_BF16)
    join_bf16(a, r32, w32, n_cu, st);
  else if (bt == AC_TYPE_F16)
    join_f16(a, r32, w32, n_cu, st);
  else
    join_f32(a, r32, w32, n_cu, st);
  return hipGetLastError();
}

bool join_bwd_means(int64_t cols) { return !bwd_whole(cols); }
void join_bwd_plan(JoinBwdArgs* b, int n_cu) {
  const JoinArgs& a = b->j;
  const bool gate = b->grad[G_GATE] != nullptr;
  b->chunks = 0;
  b->rows_per = 1;
  b->parts = 0;
  b->sections = 0;
  b->group = 1;
  for (int k = 0; k < G_COUNT; ++k) b->section[k] = -1;
  if (a.rows > 0) {
    // workgroups: eight waves a CU; of the long rows' column sums four workgroups a CU.
    // (Half as many and twice as many, forward and backward pass of bf16: 8192 x 2048 91
    // and 89 us against 78, 20000 x 768 112 and 102 against 88; twice as many of 8192 x
    // 4096 152 against 145.)
    const int64_t wide = (a.cols + 2047) / 2048, four = 4 * n_cu / wide;
    const int64_t most = !bwd_whole(a.cols) ? (four > 32 ? four : 32) : a.cols > 2048 ? n_cu : a.cols > 1024 || a.cols <= 512 ? 2 * n_cu : 4 * n_cu;
    // rows that keep a workgroup's waves at work, or are worth a partial row
    const int64_t least = a.cols <= 512 || !bwd_whole(a.cols) ? 8 : 1;
    const int64_t groups = gate ? a.rows / a.per : 1, per = gate ? a.per : a.rows;
    b->group = per;
    if (gate && (a.per == 1 || groups >= most)) {
      const int64_t n = (groups + most - 1) / most;  // groups of a workgroup
      b->rows_per = n * per;
      if (a.per == 1 && b->rows_per < least) b->rows_per = least;
      b->parts = (int)((a.rows + b->rows_per - 1) / b->rows_per);
    } else {
      int64_t chunks = most / groups;
      if (chunks > (per + least - 1) / least) chunks = (per + least - 1) / least;
      if (chunks < 1) chunks = 1;
      b->rows_per = (per + chunks - 1) / chunks;
      b->chunks = (int)((per + b->rows_per - 1) / b->rows_per);
      b->parts = (int)(groups * b->chunks);
    }
  }
  for (int k = 0; k < G_COUNT; ++k)
    if (b->grad[k] && (k != G_GATE || b->chunks > 0 || a.rows == 0)) b->section[k] = b->sections++;
}

hipError_t launch_join_bwd(const JoinBwdArgs& b, int rt, int bt, int wt, int n_cu, hipStream_t st, int* launches) {
  *launches = 0;
  if (b.j.cols <= 0) return hipSuccess;
  if (b.sections > 0 && b.parts > 0 && !b.part) return hipErrorInvalidValue;
  const bool r32 = rt == AC_TYPE_F32, w32 = wt == AC_TYPE_F32;
  *launches = bt == AC_TYPE_BF16  ? join_bwd_bf16(b, r32, w32, n_cu, st)
              : bt == AC_TYPE_F16 ? join_bwd_f16(b, r32, w32, n_cu, st)
                                  : join_bwd_f32(b, r32, w32, n_cu, st);
  return hipGetLastError();
}
#endif

}  // namespace ac
