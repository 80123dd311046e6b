// gfx950 kernels of the gated feed-forward block
//   G = X Wg, U = X Wu, H = act(G) * U, Y = H Wd
// and its backward pass
//   dH = dY Wd^T, dU = dH * act(G), dG = dH * U * act'(G),
//   dX = dG Wg^T + dU Wu^T, dWg = X^T dG, dWu = X^T dU, dWd = H^T dY,
// on the direct-to-LDS tile (dl_pipeline.h, dl_main_loop.inc):
//
//   k_gated    both projections in one tile: its columns are BN/2 features
//              of Wg and the same of Wu, in two halves of the B stage, a
//              wave's fragments alternating between them, so that a lane
//              holds G and U of the same element and H leaves the tile
//              without them having been anywhere. (Two products and an
//              elementwise kernel write and read G and U once more: 2 x 8
//              bytes an element of H in fp32.)
//   k_dgate    dH, turned into dG and dU before it leaves the tile.
//   k_multi    up to three products of one depth in one launch (the three
//              weight gradients: 3 x 896 tiles fill 256 CUs better than three
//              launches of 3.5 rounds each), each with an optional second
//              segment of K (dX: one sum over both products, no partial dX
//              written and read), split along K where tiles are few.
//   k_rows     few rows (decode) against weights stored column by column: 16
//              features a workgroup, whole K, no partial sums: the projections
//              with the activation in one launch, Y in another.
//   k_gated_sum, k_dgate_sum, k_plain_sum
//              add the partial sums of a split in their order and apply what
//              the tile's epilogue would have.
//
// Products, sums and the activation are fp32; H, G, U, dG and dU are rounded
// once to the 16-bit input format: H, dG and dU because the matrix instructions
// of their products read that format, G and U because a training step keeps them
// from the forward to the backward pass (in fp32 8 M F bytes more traffic). dX, dWg
// and dWu are so 1.8 times as far from their 64-bit values as the rounding of
// the result alone would leave them.
//
// Bound by matrix instructions from some hundred rows on, by the weights' bytes
// below. Measured, bf16, linear layers' weights, 4096 x 4096 x 14336 (M, D, F): k_gated
// 788 us (1.22 PFLOP/s), Y 387 (1.24), k_dgate 539 (0.89: its epilogue reads G and U
// and writes dG and dU, alone on its CU), dX 709 (1.36), the three weight gradients
// 1193 (1.21); a plain product of 8192^3 reaches 1.4 to 1.5. 16 rows: gate and up 52
// us (4.5 TB/s).
//
// Epilogues go through an fp32 slab per wave (32 rows, 16-byte chunks XORed
// with the row so that neither side conflicts), from which a lane takes eight
// consecutive columns: every global access is 16 bytes a lane, 128 or 256
// contiguous bytes a row.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernel_args.h"
#include "ops.h"

#ifndef AC_INPUT_F16
#define AC_INPUT_F16 0
#endif
#ifndef AC_FFN_PART
#define AC_FFN_PART 0
#endif

namespace ac {
#if AC_INPUT_F16
namespace f16 {
#endif

#include "device_common.h"

namespace {

#include "dl_pipeline.h"
#include "tile_ops.h"

// ---- activations (adaptcore_activation), fp32
// (the hardware's exponential and reciprocal: some units of 2^-24 and |x| 2^-24 of
// the value, against the 2^-12 or more of the 16-bit results; the exact forms are
// a dozen instructions more an element in epilogues that nothing overlaps)
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
constexpr float GELU_K = 0.7978845608028654f, GELU_A = 0.044715f;  // sqrt(2 / pi)
constexpr float SQRT_HALF = 0.7071067811865476f, INV_SQRT_2PI = 0.3989422804014327f;

__device__ __forceinline__ void act8(int kind, const float (&x)[8], float (&a)[8]) {
  if (kind == AC_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = x[e] * sigmoid(x[e]);
  } else if (kind == AC_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = 0.5f * x[e] * (1.0f + erff(x[e] * SQRT_HALF));
  } else {  // 0.5 (1 + tanh z) = sigmoid(2 z)
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = x[e] * sigmoid(2.0f * GELU_K * x[e] * (1.0f + GELU_A * x[e] * x[e]));
  }
}
__device__ __forceinline__ float act1(int kind, float x) {
  if (kind == AC_ACT_SILU) return x * sigmoid(x);
  if (kind == AC_ACT_GELU) return 0.5f * x * (1.0f + erff(x * SQRT_HALF));
  return x * sigmoid(2.0f * GELU_K * x * (1.0f + GELU_A * x * x));
}
// the activation and its derivative
__device__ __forceinline__ void act8_grad(int kind, const float (&x)[8], float (&a)[8], float (&d)[8]) {
  if (kind == AC_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float s = sigmoid(x[e]);
      a[e] = x[e] * s;
      d[e] = s * (1.0f + x[e] * (1.0f - s));
    }
  } else if (kind == AC_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float c = 0.5f * (1.0f + erff(x[e] * SQRT_HALF));
      a[e] = x[e] * c;
      d[e] = c + x[e] * INV_SQRT_2PI * __expf(-0.5f * x[e] * x[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // (bounded: the last factor must not be infinite where s (1 - s) is zero)
      const float x2 = fminf(x[e] * x[e], 1e30f), s = sigmoid(2.0f * GELU_K * x[e] * (1.0f + GELU_A * x2));
      a[e] = x[e] * s;
      d[e] = s + x[e] * s * (1.0f - s) * (2.0f * GELU_K * (1.0f + 3.0f * GELU_A * x2));
    }
  }
}

// ---- operand tiles of both projections: B's stage holds BN/2 columns of Wg,
// then the same of Wu
template <int BM, int BN, int BK, int S, int LAY>
struct DlDual : Dl<BM, BN, BK, S, LAY> {
  typedef DlOp<BN / 2, BK, (LAY & 2) != 0> OH;
  static constexpr int HALF = OH::BYTES;
  static_assert(2 * OH::NI == Dl<BM, BN, BK, S, LAY>::NIB, "two halves of the B stage");
};
template <class G>
struct DualTile {
  LoadPlan<G, typename G::OA, typename G::OH> l;
  const char* up;
  int64_t K;
  int kA, kB;
  __device__ __forceinline__ void init(const GatedArgs& g, int64_t m0, int64_t f0) {
    l.init(g.X, g.ldx, m0, g.M - m0, g.Wg, g.ldw, f0, g.eF - f0);
    up = reinterpret_cast<const char*>(g.Wu + f0 * (G::OH::KC ? g.ldw : 1));
    kA = (int)g.kX;
    kB = (int)g.kW;
    K = 0;
  }
};
template <class G>
struct DualLoads {
  const char* pa;
  const char* pg;
  const char* pu;
  int remA, remB;
  char* sA;
  char* sB;
  __device__ __forceinline__ void start(const DualTile<G>& t, int64_t, int64_t) {
    pa = t.l.baseA;
    pg = t.l.baseB;
    pu = t.up;
    remA = t.kA;
    remB = t.kB;
  }
  __device__ __forceinline__ void next(const DualTile<G>& t) {
    pa += G::BK * t.l.stepA;
    pg += G::BK * t.l.stepB;
    pu += G::BK * t.l.stepB;
    remA -= G::BK;
    remB -= G::BK;
  }
  __device__ __forceinline__ void issue(const DualTile<G>& t, int q) const {
    constexpr int NH = G::OH::NI;
    if (q < G::NIA)
      t.l.load_a(pa, remA, sA, q);
    else if (q < G::NIA + NH)
      t.l.load_b(pg, remB, sB, q - G::NIA);
    else
      t.l.load_b(pu, remB, sB + G::HALF, q - G::NIA - NH);
  }
};
// fragment j of a wave: 32 features of Wg (even j) or the same of Wu (odd)
template <class G>
struct DualAddrs {
  FragAddr<typename G::OA, G::BK, G::TM> a;
  struct B {
    FragAddr<typename G::OH, G::BK, G::TN / 2> h;
    __device__ __forceinline__ void init(int e0) { h.init(e0 / 2); }
    __device__ __forceinline__ u32x4 read(const char* st, int ks, int j) const {
      return h.read(st + (j & 1) * G::HALF, ks, j >> 1);
    }
  } b;
};

template <int BM, int BN, int BK, int S, int LAY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_gated(GatedArgs g) {
  typedef DlDual<BM, BN, BK, S, LAY> G;
  typedef DualLoads<G> Loads;
  typedef DualAddrs<G> Addrs;
  constexpr bool RG = false;
  AC_DL_STAGES(G);
  int tm, tn;
  tile_coords(xcd_remap(blockIdx.x, g.tiles_m * g.tiles_n), g.tiles_m, g.tiles_n, 1, tm, tn);
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  const int64_t m0 = (int64_t)tm * BM, f0 = (int64_t)tn * (BN / 2);
  const int64_t kbeg = 0;
  const int nk = (int)((g.kX + G::BK - 1) / G::BK);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave / G::WN, wc = wave % G::WN;
  DualTile<G> t;
  t.init(g, m0, f0);
#include "dl_main_loop.inc"

  stage_barrier<0>();  // no wave reads the stages any more, no load into them is in flight
  const Slab<G::WTN> s = {slab_of<G>(wave, lA0, lA1, lA2, lB0, lB1, lB2, lB3)};
  constexpr int HW = G::WTN / 2, LPR = HW / 8;  // features of a wave, lanes per row
  const int64_t rbase = m0 + wr * G::WTM, fb = f0 + wc * HW + (lane % LPR) * 8;
#pragma unroll
  for (int i = 0; i < G::TM; ++i) {
    slab_fill<G>(s, acc[i], [](int j) { return (j & 1) * HW + 32 * (j >> 1); });
#pragma unroll 1
    for (int r = lane / LPR; r < 32; r += 64 / LPR) {
      const int64_t row = rbase + 32 * i + r;
      float gv[8], uv[8], h[8];
      s.get(r, lane % LPR, gv);
      s.get(r, HW / 8 + lane % LPR, uv);
      act8(g.act, gv, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] *= uv[e];
      if (row < g.M && fb < g.F) {
        const u32x4 hv = pack8(h);
        put8(g.H + row * g.ldh, fb, g.F, hv);
        // (whole chunks: no feature past F has a weight, so its H is zero)
        if (g.H2) *reinterpret_cast<u32x4*>(g.H2 + row * g.ldh2 + fb) = hv;
        if (g.G) {
          put8(g.G + row * g.ldg, fb, g.F, pack8(gv));
          put8(g.U + row * g.ldg, fb, g.F, pack8(uv));
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // fragment row by fragment row: bounded live registers
  }
}

// dG, dU of eight elements from dH and the saved G, U
__device__ __forceinline__ void dgate8(int act, const float (&dh)[8], u32x4 gv, u32x4 uv, u32x4& dg, u32x4& du) {
  float g[8], u[8], a[8], d[8];
  values8(gv, g);
  values8(uv, u);
  act8_grad(act, g, a, d);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    a[e] *= dh[e];
    d[e] *= dh[e] * u[e];
  }
  dg = pack8(d);
  du = pack8(a);
}

template <int BM, int BN, int BK, int S, int LAY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_dgate(MultiArgs a, DgateArgs e) {
  typedef Dl<BM, BN, BK, S, LAY> G;
  typedef SegLoads<G> Loads;
  typedef FragAddrs<G> Addrs;
  constexpr bool RG = false;
  AC_DL_STAGES(G);
  const MultiProd& p = a.p[0];
  int tm, tn;
  tile_coords(xcd_remap(blockIdx.x, p.tiles_m * p.tiles_n), p.tiles_m, p.tiles_n, 1, tm, tn);
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int64_t kbeg = 0;
  const int nk = a.blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave / G::WN, wc = wave % G::WN;
  SegTile<G> t;
  t.init(p, m0, n0, a.seg, nk);
#include "dl_main_loop.inc"

  constexpr int LPR = G::WTN / 8, RPP = 64 / LPR, NP = 32 / RPP;  // lanes per row, rows per pass, passes
  const int64_t rbase = m0 + wr * G::WTM + lane / LPR, cb = n0 + wc * G::WTN + (lane % LPR) * 8;
  // G and U of a fragment row are loaded while the one before is worked on
  u32x4 gv[2][NP], uv[2][NP];
  auto fetch = [&](int i) {
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int64_t row = rbase + 32 * i + q * RPP;
      gv[i & 1][q] = uv[i & 1][q] = u32x4{};
      if (row < p.M && cb < p.N) {
        gv[i & 1][q] = get8(e.G + row * e.ldg, cb, p.N);
        uv[i & 1][q] = get8(e.U + row * e.ldg, cb, p.N);
      }
    }
  };
  fetch(0);
  stage_barrier<0>();
  const Slab<G::WTN> s = {slab_of<G>(wave, lA0, lA1, lA2, lB0, lB1, lB2, lB3)};
#pragma unroll
  for (int i = 0; i < G::TM; ++i) {
    if (i + 1 < G::TM) fetch(i + 1);
    slab_fill<G>(s, acc[i], [](int j) { return 32 * j; });
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int64_t row = rbase + 32 * i + q * RPP;
      float dh[8];
      s.get(q * RPP + lane / LPR, lane % LPR, dh);
      u32x4 dg, du;
      dgate8(e.act, dh, gv[i & 1][q], uv[i & 1][q], dg, du);
      // (the columns up to the next multiple of 8 exist in dG and dU and must
      // hold zeros, which is what dH, G and U of no feature give)
      if (row < p.M && cb < p.N) {
        __builtin_memcpy(e.dG + row * e.ldd + cb, &dg, 16);
        __builtin_memcpy(e.dU + row * e.ldd + cb, &du, 16);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <int BM, int BN, int BK, int S, int LAY, int OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_multi(MultiArgs a) {
  typedef Dl<BM, BN, BK, S, LAY> G;
  typedef SegLoads<G> Loads;
  typedef FragAddrs<G> Addrs;
  constexpr bool RG = false;
  AC_DL_STAGES(G);
  const int mblock = blockIdx.x, mblocks = gridDim.x;
#include "multi_tile.inc"
}

#if AC_FFN_PART == 0
// ---- few rows (MT * 16 at most), B stored as rows of K: C = A B (GATED:
// both products and their H). A workgroup takes 16 columns of B; its SW waves
// take 64 k each in turn, straight from memory into matrix operands: a lane
// loads two 16-byte pieces of a column, 64 bytes apart, four lanes a line of it,
// one piece for each of two instructions of 32 k. Any alignment. B is read once;
// A, small, by every workgroup from the caches.
//
// 16 x 4096 x 14336: both projections 2 x 117 MB; with K split over
// workgroups and partial sums (k_multi, k_gated_sum) the launch boundary and the
// sums' latency cost 5 us each.
template <int MT, int SW, bool GATED>
__global__ __launch_bounds__(64 * SW) __attribute__((amdgpu_waves_per_eu(4, 4))) void k_rows(RowsArgs g) {
  constexpr int NB = GATED ? 2 : 1, U = GATED && MT > 1 ? 1 : 2;
  __shared__ __attribute__((aligned(16))) float part[SW * NB * MT * 256];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, kq = (lane >> 4) * 8;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const uint16_t* b[NB];
  const uint16_t* x[MT];
  bool in[MT];
#pragma unroll
  for (int j = 0; j < NB; ++j) b[j] = (j ? g.B2 : g.B) + min(n0 + i16, g.N - 1) * g.ldb;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    in[m] = m * 16 + i16 < g.M;
    x[m] = g.A + min((int64_t)(m * 16 + i16), g.M - 1) * g.lda;
  }
  f32x4 acc[NB][MT];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[j][m] = f32x4{};
  // U steps at a time, the next ones' loads issued before this one's products. A
  // batch's later steps may not exist: zeros then, so that a wave's last step needs
  // no trip to memory of its own (block of 27 x 2048 x 1536: 15.7 us with, 14.8
  // without).
  const int64_t whole = g.K / 64;
  struct Batch {
    u32x4 b[U][NB][2], x[U][MT][2];
  };
  auto load = [&](Batch& v, int64_t s) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = (s + u * SW) * 64 + kq;
#pragma unroll
      for (int j = 0; j < NB; ++j) v.b[u][j][0] = v.b[u][j][1] = u32x4{};
#pragma unroll
      for (int m = 0; m < MT; ++m) v.x[u][m][0] = v.x[u][m][1] = u32x4{};
      if (u > 0 && s + u * SW >= whole) continue;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) v.b[u][j][h] = load16(b[j] + k + 32 * h);
#pragma unroll
      for (int m = 0; m < MT; ++m)
        if (in[m]) {
#pragma unroll
          for (int h = 0; h < 2; ++h) v.x[u][m][h] = load16(x[m] + k + 32 * h);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](const Batch& v) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[j][m] = mfma16(v.b[u][j][h], v.x[u][m][h], acc[j][m]);
    __builtin_amdgcn_sched_barrier(0);
  };
  int64_t s = w;
  Batch p, q;
  if (s < whole) {
    load(p, s);
    for (;;) {
      s += U * SW;
      const bool more = s < whole;
      if (more) load(q, s);
      multiply(p);
      if (!more) break;
      s += U * SW;
      const bool again = s < whole;
      if (again) load(p, s);
      multiply(q);
      if (!again) break;
    }
  }
  // the step that K ends in
  if (whole * 64 < g.K && whole % SW == w) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t k = whole * 64 + kq + 32 * h;
      u32x4 xv[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) xv[m] = load_row(x[m], k, g.K);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const u32x4 bv = load_row(b[j], k, g.K);
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[j][m] = mfma16(bv, xv[m], acc[j][m]);
      }
    }
  }
  // a lane has row i16 and four columns of it; the waves' sums are added in
  // their order
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m)
      *reinterpret_cast<f32x4*>(part + ((w * NB + j) * MT + m) * 256 + i16 * 16 + (lane >> 4) * 4) = acc[j][m];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += 64 * SW) {
    const int64_t row = i >> 4, c = n0 + (i & 15);
    if (row >= g.M || c >= g.N) continue;
    float v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      v[j] = part[j * MT * 256 + i];
#pragma unroll
      for (int q = 1; q < SW; ++q) v[j] += part[(q * NB + j) * MT * 256 + i];
    }
    if constexpr (GATED) {
      static_cast<uint16_t*>(g.C)[row * g.ldc + c] = to16(act1(g.act, v[0]) * v[NB - 1]);
      if (g.G) {
        g.G[row * g.ldg + c] = to16(v[0]);
        g.U[row * g.ldg + c] = to16(v[NB - 1]);
      }
    } else {
      static_cast<uint16_t*>(g.C)[row * g.ldc + c] = to16(v[0]);
    }
  }
}
template <int MT, bool GATED>
hipError_t launch_rows(const RowsArgs& g, hipStream_t st) {
  const dim3 grid((unsigned)((g.N + 15) / 16));
  // As many waves as leave room for every workgroup at once (16 waves a CU) and
  // need no second batch of two steps of 64 k: one row through a block of 640 x 896
  // 7.6 us with 4 waves for its 10 and 14 steps, 6.0 with 8; of 1024 x 1024 6.8
  // with 8 for its 16, 7.1 with 16.
  const int64_t steps = (g.K + 63) / 64;
  if (grid.x <= 256 && steps > 16)
    hipLaunchKernelGGL((k_rows<MT, 16, GATED>), grid, dim3(1024), 0, st, g);
  else if (grid.x <= 512 && steps > 8)
    hipLaunchKernelGGL((k_rows<MT, 8, GATED>), grid, dim3(512), 0, st, g);
  else
    hipLaunchKernelGGL((k_rows<MT, 4, GATED>), grid, dim3(256), 0, st, g);
  return hipGetLastError();
}

#if !AC_INPUT_F16
// Zero-padded copies of several matrices (rows of cols to rows of ld_dst, a
// multiple of 8, 16-byte aligned) in one launch: a training step of a block with
// odd sizes makes ten, which took 5 us each for the launch alone. A workgroup
// copies `per` rows of one of them, 16 bytes a thread, 256 >> lg rows at a time.
__global__ __launch_bounds__(256) void k_pad_many(PadArgs a) {
  int b = blockIdx.x, m = 0;
  while (b >= a.m[m].blocks) b -= a.m[m++].blocks;
  const PadMat& p = a.m[m];
  const int tx = threadIdx.x & ((1 << p.lg) - 1), ty = threadIdx.x >> p.lg;
  const int64_t end = min((int64_t)(b + 1) * p.per, p.rows);
  for (int64_t r = (int64_t)b * p.per + ty; r < end; r += 256 >> p.lg)
    for (int64_t c = tx * 8; c < p.ld_dst; c += 8 << p.lg) {
      const u32x4 v = get8(p.src + r * p.ld_src, c, p.cols);
      *reinterpret_cast<u32x4*>(p.dst + r * p.ld_dst + c) = v;
    }
}
#endif

__global__ __launch_bounds__(256) void k_gated_sum(MultiArgs a, GatedArgs g) {
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= g.F) return;
  for (int64_t row = blockIdx.y; row < g.M; row += gridDim.y) {
    float gv[8], uv[8], h[8];
    part_sum(a.p[0], a.pk, row, c, gv);
    part_sum(a.p[1], a.pk, row, c, uv);
    act8(g.act, gv, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] *= uv[e];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = c + e < g.F ? h[e] : 0.f;
    put8(g.H + row * g.ldh, c, g.F, pack8(h));
    if (g.H2) *reinterpret_cast<u32x4*>(g.H2 + row * g.ldh2 + c) = pack8(h);
    if (g.G) {
      put8(g.G + row * g.ldg, c, g.F, pack8(gv));
      put8(g.U + row * g.ldg, c, g.F, pack8(uv));
    }
  }
}
__global__ __launch_bounds__(256) void k_dgate_sum(MultiArgs a, DgateArgs e) {
  const MultiProd& p = a.p[0];
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= p.N) return;
  for (int64_t row = blockIdx.y; row < p.M; row += gridDim.y) {
    float dh[8];
    part_sum(p, a.pk, row, c, dh);
#pragma unroll
    for (int i = 0; i < 8; ++i) dh[i] = c + i < p.N ? dh[i] : 0.f;
    u32x4 dg, du;
    dgate8(e.act, dh, get8(e.G + row * e.ldg, c, p.N), get8(e.U + row * e.ldg, c, p.N), dg, du);
    __builtin_memcpy(e.dG + row * e.ldd + c, &dg, 16);
    __builtin_memcpy(e.dU + row * e.ldd + c, &du, 16);
  }
}
template <bool OUT16>
__global__ __launch_bounds__(256) void k_plain_sum(MultiArgs a) {
  const MultiProd& p = a.p[blockIdx.z];
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= p.N) return;
  for (int64_t row = blockIdx.y; row < p.M; row += gridDim.y) {
    float v[8];
    part_sum(p, a.pk, row, c, v);
    if constexpr (OUT16) {
      put8(static_cast<uint16_t*>(p.C) + row * p.ldc, c, p.N, pack8(v));
    } else {
      put8f(static_cast<float*>(p.C) + row * p.ldc, c, p.N, v);
    }
  }
}
dim3 sum_grid(int64_t rows, int64_t cols, int z) {
  return dim3((unsigned)((cols + 2047) / 2048), (unsigned)(rows < 32768 ? rows : 32768), z);
}
#endif

}  // namespace

// ---- launchers. The tile kernels are compiled in parts (AC_FFN_PART), one
// per tile, so that the build runs in parallel.
template <int BM, int BN, int BK, int S>
hipError_t launch_multi(const MultiArgs& a, int lay, int out, hipStream_t st) {
  int tiles = 0;
  for (int i = 0; i < a.n; ++i) tiles += a.p[i].tiles_m * a.p[i].tiles_n;
  const dim3 grid(tiles, a.pk), block(256);
  const int o = a.pk > 1 ? DL_PARTIAL : out;
#define AC_MULTI(L, O)                                                                  \
  if (lay == L && o == O) {                                                             \
    hipLaunchKernelGGL((k_multi<BM, BN, BK, S, L, O>), grid, block, 0, st, a);          \
    return hipGetLastError();                                                           \
  }
  AC_MULTI(0, DL_BF16)
  AC_MULTI(0, DL_PARTIAL)
  AC_MULTI(2, DL_BF16)
  AC_MULTI(2, DL_PARTIAL)
  if constexpr (BM >= 128) {
    AC_MULTI(1, DL_BF16)
    AC_MULTI(1, DL_F32)
    AC_MULTI(1, DL_PARTIAL)
  }
#undef AC_MULTI
  return hipErrorInvalidValue;
}
template <int BM, int BN, int BK, int S>
hipError_t launch_dgate(const MultiArgs& a, const DgateArgs& e, int lay, hipStream_t st) {
  const dim3 grid(a.p[0].tiles_m * a.p[0].tiles_n), block(256);
  if (lay == 0)
    hipLaunchKernelGGL((k_dgate<BM, BN, BK, S, 0>), grid, block, 0, st, a, e);
  else
    hipLaunchKernelGGL((k_dgate<BM, BN, BK, S, 2>), grid, block, 0, st, a, e);
  return hipGetLastError();
}
template <int BM, int BN, int BK, int S>
hipError_t launch_gated(const GatedArgs& g, int lay, hipStream_t st) {
  const dim3 grid(g.tiles_m * g.tiles_n), block(256);
  if (lay == 2) {
    hipLaunchKernelGGL((k_gated<BM, BN, BK, S, 2>), grid, block, 0, st, g);
    return hipGetLastError();
  }
  if constexpr (BN >= 256) {  // (rows of k: 128 features of each weight at least)
    hipLaunchKernelGGL((k_gated<BM, BN, BK, S, 0>), grid, block, 0, st, g);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}
#define FFN_MULTI(a, b, c, d) template hipError_t launch_multi<a, b, c, d>(const MultiArgs&, int, int, hipStream_t);
#define FFN_DGATE(a, b, c, d) \
  template hipError_t launch_dgate<a, b, c, d>(const MultiArgs&, const DgateArgs&, int, hipStream_t);
#define FFN_GATED(a, b, c, d) template hipError_t launch_gated<a, b, c, d>(const GatedArgs&, int, hipStream_t);

#if AC_FFN_PART == 1
FFN_MULTI(256, 256, 64, 2)
#elif AC_FFN_PART == 2
FFN_DGATE(256, 256, 64, 2)
FFN_GATED(256, 256, 64, 2)
#elif AC_FFN_PART == 3
FFN_MULTI(128, 256, 64, 3)
#elif AC_FFN_PART == 4
FFN_GATED(128, 256, 64, 3)
#elif AC_FFN_PART == 5
FFN_MULTI(128, 128, 64, 2)
FFN_DGATE(128, 128, 64, 2)
FFN_GATED(128, 128, 64, 2)
#elif AC_FFN_PART == 6
FFN_MULTI(128, 128, 64, 3)
FFN_DGATE(128, 128, 64, 3)
FFN_GATED(128, 128, 64, 3)
#elif AC_FFN_PART == 7
FFN_MULTI(64, 256, 64, 4)
FFN_MULTI(32, 256, 64, 4)
FFN_MULTI(32, 128, 64, 4)
#else
extern FFN_MULTI(256, 256, 64, 2) extern FFN_MULTI(128, 256, 64, 3) extern FFN_MULTI(128, 128, 64, 2)
extern FFN_MULTI(128, 128, 64, 3) extern FFN_DGATE(128, 128, 64, 3) extern FFN_GATED(128, 128, 64, 3)
extern FFN_MULTI(64, 256, 64, 4) extern FFN_MULTI(32, 256, 64, 4) extern FFN_MULTI(32, 128, 64, 4)
extern FFN_DGATE(256, 256, 64, 2) extern FFN_DGATE(128, 128, 64, 2)
extern FFN_GATED(256, 256, 64, 2) extern FFN_GATED(128, 256, 64, 3) extern FFN_GATED(128, 128, 64, 2)

hipError_t ffn_multi(const FfnTile& t, const MultiArgs& a, int lay, int out, hipStream_t st) {
  if (a.n < 1 || a.n > 3 || a.pk < 1 || a.kper < 1 || (int64_t)a.kper * a.pk < a.blocks) return hipErrorInvalidValue;
  const auto is = [&](int bm, int bn, int stages) { return t.bm == bm && t.bn == bn && t.stages == stages; };
  if (is(256, 256, 2)) return launch_multi<256, 256, 64, 2>(a, lay, out, st);
  if (is(128, 256, 3)) return launch_multi<128, 256, 64, 3>(a, lay, out, st);
  if (is(128, 128, 2)) return launch_multi<128, 128, 64, 2>(a, lay, out, st);
  if (is(128, 128, 3)) return launch_multi<128, 128, 64, 3>(a, lay, out, st);
  if (is(64, 256, 4)) return launch_multi<64, 256, 64, 4>(a, lay, out, st);
  if (is(32, 256, 4)) return launch_multi<32, 256, 64, 4>(a, lay, out, st);
  if (is(32, 128, 4)) return launch_multi<32, 128, 64, 4>(a, lay, out, st);
  return hipErrorInvalidValue;
}
hipError_t ffn_dgate(const FfnTile& t, const MultiArgs& a, const DgateArgs& e, int lay, hipStream_t st) {
  const auto is = [&](int bm, int bn, int stages) { return t.bm == bm && t.bn == bn && t.stages == stages; };
  if (is(256, 256, 2)) return launch_dgate<256, 256, 64, 2>(a, e, lay, st);
  if (is(128, 128, 2)) return launch_dgate<128, 128, 64, 2>(a, e, lay, st);
  if (is(128, 128, 3)) return launch_dgate<128, 128, 64, 3>(a, e, lay, st);
  return hipErrorInvalidValue;
}
hipError_t ffn_gated(const FfnTile& t, const GatedArgs& g, int lay, hipStream_t st) {
  const auto is = [&](int bm, int bn, int stages) { return t.bm == bm && t.bn == bn && t.stages == stages; };
  if (is(256, 256, 2)) return launch_gated<256, 256, 64, 2>(g, lay, st);
  if (is(128, 256, 3)) return launch_gated<128, 256, 64, 3>(g, lay, st);
  if (is(128, 128, 2)) return launch_gated<128, 128, 64, 2>(g, lay, st);
  if (is(128, 128, 3)) return launch_gated<128, 128, 64, 3>(g, lay, st);
  return hipErrorInvalidValue;
}
#if !AC_INPUT_F16
}  // namespace ac
namespace ac {
hipError_t launch_pad_many(PadArgs a, hipStream_t st) {
  int64_t blocks = 0;
  for (int i = 0; i < a.n; ++i) {
    PadMat& p = a.m[i];
    if (p.ld_dst < p.cols || p.ld_src < p.cols || p.ld_dst % 8 != 0 || p.rows < 1 || p.cols < 1 ||
        (reinterpret_cast<uintptr_t>(p.dst) & 15) != 0)
      return hipErrorInvalidValue;
    const int64_t chunks = p.ld_dst / 8;  // of a row
    p.lg = 0;
    while (p.lg < 8 && (1 << p.lg) < chunks) ++p.lg;
    // about eight chunks a thread
    p.per = (int)(2048 / chunks > 256 >> p.lg ? 2048 / chunks : 256 >> p.lg);
    const int64_t n = (p.rows + p.per - 1) / p.per;
    blocks += n;
    if (blocks >= (1LL << 31) / 256) return hipErrorInvalidValue;
    p.blocks = (int)n;
  }
  if (blocks > 0) hipLaunchKernelGGL(k_pad_many, dim3((unsigned)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}
#endif
hipError_t ffn_rows(const RowsArgs& g, bool gated, hipStream_t st) {
  if (g.M < 1 || g.M > FFN_ROWS_MAX || g.N < 1 || g.K < 1) return hipErrorInvalidValue;
  if (g.M <= 16) return gated ? launch_rows<1, true>(g, st) : launch_rows<1, false>(g, st);
  return gated ? launch_rows<2, true>(g, st) : launch_rows<2, false>(g, st);
}
hipError_t ffn_gated_sum(const MultiArgs& a, const GatedArgs& g, hipStream_t st) {
  hipLaunchKernelGGL(k_gated_sum, sum_grid(g.M, g.F, 1), dim3(256), 0, st, a, g);
  return hipGetLastError();
}
hipError_t ffn_dgate_sum(const MultiArgs& a, const DgateArgs& e, hipStream_t st) {
  hipLaunchKernelGGL(k_dgate_sum, sum_grid(a.p[0].M, a.p[0].N, 1), dim3(256), 0, st, a, e);
  return hipGetLastError();
}
hipError_t ffn_plain_sum(const MultiArgs& a, int out, hipStream_t st) {
  int64_t rows = 0, cols = 0;
  for (int i = 0; i < a.n; ++i) {
    rows = rows > a.p[i].M ? rows : a.p[i].M;
    cols = cols > a.p[i].N ? cols : a.p[i].N;
  }
  if (out == 1)
    hipLaunchKernelGGL((k_plain_sum<true>), sum_grid(rows, cols, a.n), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_plain_sum<false>), sum_grid(rows, cols, a.n), dim3(256), 0, st, a);
  return hipGetLastError();
}
#endif

#if AC_INPUT_F16
}  // namespace f16
#endif
}  // namespace ac
