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
//   k_gated_sum, k_dgate_sum, k_plain_sum
//              add the partial sums of a split in their order and apply what
//              the tile's epilogue would have.
//
// Products, sums and the activation are fp32; H, G, U, dG and dU are rounded
// once to the 16-bit input format, the format their product reads them in.
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
      const float x2 = x[e] * x[e], s = sigmoid(2.0f * GELU_K * x[e] * (1.0f + GELU_A * x2));
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
        put8(g.H + row * g.ldh, fb, g.F, pack8(h));
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
    put8(g.H + row * g.ldh, c, g.F, pack8(h));
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
  if (lay == 0)
    hipLaunchKernelGGL((k_gated<BM, BN, BK, S, 0>), grid, block, 0, st, g);
  else
    hipLaunchKernelGGL((k_gated<BM, BN, BK, S, 2>), grid, block, 0, st, g);
  return hipGetLastError();
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
FFN_DGATE(128, 256, 64, 3)
FFN_GATED(128, 256, 64, 3)
#elif AC_FFN_PART == 5
FFN_MULTI(128, 128, 64, 2)
FFN_DGATE(128, 128, 64, 2)
#elif AC_FFN_PART == 6
FFN_MULTI(64, 256, 64, 4)
FFN_MULTI(32, 256, 64, 4)
FFN_MULTI(32, 128, 64, 4)
#else
extern FFN_MULTI(256, 256, 64, 2) extern FFN_MULTI(128, 256, 64, 3) extern FFN_MULTI(128, 128, 64, 2)
extern FFN_MULTI(64, 256, 64, 4) extern FFN_MULTI(32, 256, 64, 4) extern FFN_MULTI(32, 128, 64, 4)
extern FFN_DGATE(256, 256, 64, 2) extern FFN_DGATE(128, 256, 64, 3) extern FFN_DGATE(128, 128, 64, 2)
extern FFN_GATED(256, 256, 64, 2) extern FFN_GATED(128, 256, 64, 3)

hipError_t ffn_multi(const FfnTile& t, const MultiArgs& a, int lay, int out, hipStream_t st) {
  if (a.n < 1 || a.n > 3 || a.pk < 1 || a.kper < 1 || (int64_t)a.kper * a.pk < a.blocks) return hipErrorInvalidValue;
  if (t.bm == 256 && t.bn == 256) return launch_multi<256, 256, 64, 2>(a, lay, out, st);
  if (t.bm == 128 && t.bn == 256) return launch_multi<128, 256, 64, 3>(a, lay, out, st);
  if (t.bm == 128 && t.bn == 128) return launch_multi<128, 128, 64, 2>(a, lay, out, st);
  if (t.bm == 64 && t.bn == 256) return launch_multi<64, 256, 64, 4>(a, lay, out, st);
  if (t.bm == 32 && t.bn == 256) return launch_multi<32, 256, 64, 4>(a, lay, out, st);
  if (t.bm == 32 && t.bn == 128) return launch_multi<32, 128, 64, 4>(a, lay, out, st);
  return hipErrorInvalidValue;
}
hipError_t ffn_dgate(const FfnTile& t, const MultiArgs& a, const DgateArgs& e, int lay, hipStream_t st) {
  if (t.bm == 256 && t.bn == 256) return launch_dgate<256, 256, 64, 2>(a, e, lay, st);
  if (t.bm == 128 && t.bn == 256) return launch_dgate<128, 256, 64, 3>(a, e, lay, st);
  if (t.bm == 128 && t.bn == 128) return launch_dgate<128, 128, 64, 2>(a, e, lay, st);
  return hipErrorInvalidValue;
}
hipError_t ffn_gated(const FfnTile& t, const GatedArgs& g, int lay, hipStream_t st) {
  if (t.bm == 256 && t.bn == 256) return launch_gated<256, 256, 64, 2>(g, lay, st);
  if (t.bm == 128 && t.bn == 256) return launch_gated<128, 256, 64, 3>(g, lay, st);
  return hipErrorInvalidValue;
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
