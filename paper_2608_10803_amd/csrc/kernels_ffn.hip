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

// Eight 16-bit values of a row from column c on; those at or past n are not
// touched (read as zero).
__device__ __forceinline__ u32x4 get8(const uint16_t* row, int64_t c, int64_t n) {
  if (c + 8 <= n) return load16(row + c);
  uint32_t h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = c + e < n ? row[c + e] : 0u;
  return u32x4{h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16)};
}
__device__ __forceinline__ void values8(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = from16((v[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (uint32_t)to16(f[2 * e]) | ((uint32_t)to16(f[2 * e + 1]) << 16);
  return v;
}
__device__ __forceinline__ void put8(uint16_t* row, int64_t c, int64_t n, u32x4 v) {
  if (c + 8 <= n) {
    __builtin_memcpy(row + c, &v, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) row[c + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
  }
}

// ---- a wave's epilogue slab: 32 rows x W fp32, chunk c (4 columns) of row r
// at c ^ r: 32 lanes writing one chunk of 32 rows, or reading a row's chunks,
// fall on distinct banks.
template <int W>
struct Slab {
  static constexpr int CH = W / 4, BYTES = 32 * W * 4;
  char* p;
  __device__ __forceinline__ void put(int row, int c, float a, float b, float d, float e) const {
    *reinterpret_cast<f32x4*>(p + row * (W * 4) + ((c ^ (row & (CH - 1))) << 4)) = f32x4{a, b, d, e};
  }
  __device__ __forceinline__ f32x4 get4(int row, int c) const {
    return *reinterpret_cast<const f32x4*>(p + row * (W * 4) + ((c ^ (row & (CH - 1))) << 4));
  }
  // columns 8 * g .. 8 * g + 7
  __device__ __forceinline__ void get(int row, int g, float (&f)[8]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 v = get4(row, 2 * g + h);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * h + e] = v[e];
    }
  }
};
// the slab of wave w: one stage buffer each (two of A's and two of B's, or
// three and one, or four of B's)
template <class G>
__device__ __forceinline__ char* slab_of(int w, char* a0, char* a1, char* a2, char* b0, char* b1, char* b2, char* b3) {
  static_assert(Slab<G::WTN>::BYTES <= G::B_BYTES && (G::S >= 4 || Slab<G::WTN>::BYTES <= G::A_BYTES), "slab");
  if constexpr (G::S >= 4)
    return w == 0 ? b0 : w == 1 ? b1 : w == 2 ? b2 : b3;
  else if constexpr (G::S == 3)
    return w == 0 ? a0 : w == 1 ? a1 : w == 2 ? a2 : b0;
  else
    return w == 0 ? a0 : w == 1 ? a1 : w == 2 ? b0 : b1;
}
template <class G>
__device__ __forceinline__ void slab_fill(const Slab<G::WTN>& s, const f32x16 (&acc)[G::TN], int col_of_j(int)) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < G::TN; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      s.put(lane & 31, col_of_j(j) / 4 + 2 * q + (lane >> 5), acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2],
            acc[j][4 * q + 3]);
}

// ---- operand tiles of a product with an optional second segment of K
template <class G>
struct SegTile {
  DlOpTile<typename G::OA, G::BK> a;
  DlOpTile<typename G::OB, G::BK> b;
  const char* a2;
  const char* b2;
  int64_t K;  // (of the register-load form, not used here)
  int kA, kB;     // k that a segment of each operand holds
  int seg, end;   // first k-block of the second segment, and past the partition
  int w;

  __device__ __forceinline__ void init(const MultiProd& p, int64_t m0, int64_t n0, int kseg, int end_block) {
    w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    a.init(p.A, p.lda, m0, p.eA - m0, w);
    b.init(p.B, p.ldb, n0, p.eB - n0, w);
    a2 = reinterpret_cast<const char*>(p.A2 + m0 * (G::OA::KC ? p.lda : 1));
    b2 = reinterpret_cast<const char*>(p.B2 + n0 * (G::OB::KC ? p.ldb : 1));
    kA = (int)p.kA;
    kB = (int)p.kB;
    seg = kseg;
    end = end_block;
    K = 0;
  }
};
template <class G>
struct SegLoads {
  const char* pa;
  const char* pb;
  int remA, remB, blk;
  char* sA;
  char* sB;
  __device__ __forceinline__ void start(const SegTile<G>& t, int64_t kbeg, int64_t) {
    blk = (int)(kbeg / G::BK);
    const bool two = blk >= t.seg;
    const int k = (two ? blk - t.seg : blk) * G::BK;
    pa = (two ? t.a2 : t.a.base) + k * t.a.kstep;
    pb = (two ? t.b2 : t.b.base) + k * t.b.kstep;
    remA = blk < t.end ? t.kA - k : 0;
    remB = blk < t.end ? t.kB - k : 0;
  }
  __device__ __forceinline__ void next(const SegTile<G>& t) {
    ++blk;
    const bool two = blk == t.seg;
    pa = two ? t.a2 : pa + G::BK * t.a.kstep;
    pb = two ? t.b2 : pb + G::BK * t.b.kstep;
    remA = two ? t.kA : remA - G::BK;
    remB = two ? t.kB : remB - G::BK;
    if (blk >= t.end) remA = remB = 0;  // past the partition: zeros, no traffic
  }
  __device__ __forceinline__ void issue(const SegTile<G>& t, int q) const {
    if (q < G::NIA)
      t.a.issue(pa, remA, sA, t.w, q);
    else
      t.b.issue(pb, remB, sB, t.w, q - G::NIA);
  }
};

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
  DlOpTile<typename G::OA, G::BK> a;
  DlOpTile<typename G::OH, G::BK> b;
  const char* up;
  int64_t K;
  int kA, kB, w;
  __device__ __forceinline__ void init(const GatedArgs& g, int64_t m0, int64_t f0) {
    w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    a.init(g.X, g.ldx, m0, g.M - m0, w);
    b.init(g.Wg, g.ldw, f0, g.eF - f0, w);
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
    pa = t.a.base;
    pg = t.b.base;
    pu = t.up;
    remA = t.kA;
    remB = t.kB;
  }
  __device__ __forceinline__ void next(const DualTile<G>& t) {
    pa += G::BK * t.a.kstep;
    pg += G::BK * t.b.kstep;
    pu += G::BK * t.b.kstep;
    remA -= G::BK;
    remB -= G::BK;
  }
  __device__ __forceinline__ void issue(const DualTile<G>& t, int q) const {
    constexpr int NH = G::OH::NI;
    if (q < G::NIA)
      t.a.issue(pa, remA, sA, t.w, q);
    else if (q < G::NIA + NH)
      t.b.issue(pg, remB, sB, t.w, q - G::NIA);
    else
      t.b.issue(pu, remB, sB + G::HALF, t.w, q - G::NIA - NH);
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
  int tile = xcd_remap(blockIdx.x, gridDim.x);
  const int n0t = a.p[0].tiles_m * a.p[0].tiles_n, n1t = a.p[1].tiles_m * a.p[1].tiles_n;
  const int which = __builtin_amdgcn_readfirstlane(tile < n0t ? 0 : tile < n0t + n1t ? 1 : 2);
  tile -= which == 0 ? 0 : which == 1 ? n0t : n0t + n1t;
  const MultiProd& p = a.p[which];
  int tm, tn;
  tile_coords(tile, p.tiles_m, p.tiles_n, 1, tm, tn);
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int beg = min((int)blockIdx.y * a.kper, a.blocks), end = min(beg + a.kper, a.blocks);
  const int64_t kbeg = (int64_t)beg * G::BK;
  const int nk = end - beg;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave / G::WN, wc = wave % G::WN;
  SegTile<G> t;
  t.init(p, m0, n0, a.seg, end);
#include "dl_main_loop.inc"

  stage_barrier<0>();
  const Slab<G::WTN> s = {slab_of<G>(wave, lA0, lA1, lA2, lB0, lB1, lB2, lB3)};
  const int64_t rbase = m0 + wr * G::WTM, cbase = n0 + wc * G::WTN;
  constexpr int PER = OUT == DL_BF16 ? 8 : 4, LPR = G::WTN / PER;  // columns of a lane, lanes per row
  const int64_t c = cbase + (lane % LPR) * PER;
#pragma unroll
  for (int i = 0; i < G::TM; ++i) {
    slab_fill<G>(s, acc[i], [](int j) { return 32 * j; });
#pragma unroll 4
    for (int r = lane / LPR; r < 32; r += 64 / LPR) {
      const int64_t row = rbase + 32 * i + r;
      if constexpr (OUT == DL_BF16) {
        float v[8];
        s.get(r, lane % LPR, v);
        if (row < p.M && c < p.N) put8(static_cast<uint16_t*>(p.C) + row * p.ldc, c, p.N, pack8(v));
      } else {
        const f32x4 v = s.get4(r, lane % LPR);
        float* dst = OUT == DL_PARTIAL ? p.part + ((int64_t)blockIdx.y * p.M + row) * p.ldp
                                       : static_cast<float*>(p.C) + row * p.ldc;
        if (row < p.M && c + 4 <= p.N) {
          __builtin_memcpy(dst + c, &v, 16);
        } else if (row < p.M) {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (c + e < p.N) dst[c + e] = v[e];
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

#if AC_FFN_PART == 0
// ---- sums over the partitions of a split product, in their order; a thread
// takes eight columns of one row (ldp is a multiple of 8, so the loads are
// whole; columns at or past N hold whatever and go nowhere)
__device__ __forceinline__ void part_sum(const MultiProd& p, int pk, int64_t row, int64_t c, float (&v)[8]) {
  const float* src = p.part + row * p.ldp + c;
  const int64_t slice = p.M * p.ldp;
  f32x4 s0 = *reinterpret_cast<const f32x4*>(src), s1 = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll 4
  for (int i = 1; i < pk; ++i) {
    s0 += *reinterpret_cast<const f32x4*>(src + i * slice);
    s1 += *reinterpret_cast<const f32x4*>(src + i * slice + 4);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = s0[e];
    v[4 + e] = s1[e];
  }
}
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
      float* dst = static_cast<float*>(p.C) + row * p.ldc + c;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < p.N) dst[e] = v[e];
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
