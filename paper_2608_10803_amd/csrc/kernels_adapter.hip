// gfx950 kernels of low-rank adapters beside a shared projection:
//   Y[i] = X[i] W + bias + T[i] up[a]^T,  T[i] = scale[a] X[i] down[a]^T,
//   a = index[i] (a row whose index is not one of the adapters has none),
// for rows of many requests in one product.
//
//   k_shrink       T, for every row. A workgroup takes 16 (or 64) rows, 16 of
//                  the rank and ONE of the adapters that the rows use: there
//                  is a workgroup per row, and it works if its row is the first
//                  of the tile with its adapter, for all the tile's rows of
//                  that adapter. So no sorting, no host knowledge of the
//                  indices, every adapter read once a tile, and all of a tile's
//                  adapters at once. K is split over the workgroup's waves.
//   k_adapter      the shared product on the direct-to-LDS tile; before its
//                  epilogue each wave adds T up^T for the adapters of its rows
//                  one after the other, with the other rows' T as zeros, from
//                  global memory (R values a row and column against K of the
//                  main loop). Y is written once.
//   k_adapter_sum  few rows: adds the partial sums of the shared product,
//                  split along K, and T up^T with FMAs. There the adapters'
//                  bytes count like the weights': each is read where it is used
//                  once, R contiguous values a column.
//
// Sums are fp32. k_adapter multiplies T by matrix instructions, so T is rounded
// to the input format there (one part in 2^9 of the adapters' share);
// k_adapter_sum keeps it in fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernel_args.h"
#include "ops.h"

#ifndef AC_INPUT_F16
#define AC_INPUT_F16 0
#endif

namespace ac {
#if AC_INPUT_F16
namespace f16 {
#endif

#include "device_common.h"

namespace {

#include "dl_pipeline.h"
#include "tile_ops.h"

// The adapter of a row, -1 where it has none.
__device__ __forceinline__ int adapter_of(const AdapterArgs& g, int64_t row) {
  const int a = row < g.M ? g.index[row] : -1;
  return a >= 0 && a < g.n ? a : -1;
}

// T: MT * 16 rows, blockIdx.x = row tile * rows + the row, blockIdx.y = 16 of
// the rank. SW waves take 32 k each in turn.
constexpr int SW = 8;
template <int MT, bool T16>
__global__ __launch_bounds__(64 * SW) void k_shrink(AdapterArgs g) {
  __shared__ float part[SW][MT * 16 * 16];
  constexpr int ROWS = MT * 16;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t m0 = (int64_t)(blockIdx.x / ROWS) * ROWS;
  const int me = blockIdx.x % ROWS;
  const int mine = lane < ROWS ? adapter_of(g, m0 + lane) : -1;
  const int a = __builtin_amdgcn_readfirstlane(__shfl(mine, me));
  if (a < 0) return;
  const uint64_t rows = __ballot(mine == a);
  if (rows & ((1ull << me) - 1)) return;  // an earlier row's workgroup has this adapter

  const int r0 = blockIdx.y * 16, i16 = lane & 15, kq = (lane >> 4) * 8;
  const uint16_t* down = g.down + a * g.stride_down + (int64_t)min(r0 + i16, g.R - 1) * g.ld_down;
  const uint16_t* x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x[m] = g.X + min(m0 + m * 16 + i16, g.M - 1) * g.ldx;
  f32x4 acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = f32x4{};
  // whole steps of 32 k, several loads in flight, then the tail
  const int64_t whole = g.K / 32;
  int64_t s = w;
  constexpr int U = MT == 1 ? 8 : 4;
  for (; s + (U - 1) * SW < whole; s += U * SW) {
    u32x4 d[U], v[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = (s + u * SW) * 32 + kq;
      d[u] = load16(down + k);
#pragma unroll
      for (int m = 0; m < MT; ++m) v[u][m] = load16(x[m] + k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m] = mfma16(v[u][m], d[u], acc[m]);
  }
  for (; s * 32 < g.K; s += SW) {
    const int64_t k = s * 32 + kq;
    const u32x4 d = get8(down, k, g.K);
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = mfma16(get8(x[m], k, g.K), d, acc[m]);
  }
  // the waves' sums, added in their order; lane: column i16, rows 4 * (lane >> 4) ..
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[w][(m * 16 + (lane >> 4) * 4 + e) * 16 + i16] = acc[m][e];
  __syncthreads();
  const float scale = g.scale ? g.scale[a] : 1.0f;
  for (int i = threadIdx.x; i < ROWS * 16; i += 64 * SW) {
    const int row = i >> 4, r = r0 + (i & 15);
    if (!((rows >> row) & 1)) continue;
    float v = part[0][i];
#pragma unroll
    for (int j = 1; j < SW; ++j) v += part[j][i];
    v = r < g.R ? v * scale : 0.f;
    if constexpr (T16)
      static_cast<uint16_t*>(g.T)[(m0 + row) * g.ldt + r] = to16(v);
    else
      static_cast<float*>(g.T)[(m0 + row) * g.ldt + r] = v;
  }
}

template <int BM, int BN, int BK, int S, int LAY, bool OUT16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_adapter(MultiArgs a, AdapterArgs g) {
  typedef Dl<BM, BN, BK, S, LAY> G;
  typedef SegLoads<G> Loads;
  typedef FragAddrs<G> Addrs;
  constexpr bool RG = false;
  AC_DL_STAGES(G);
  const MultiProd& p = a.p[0];
  int tm, tn;
  tile_coords(xcd_remap(blockIdx.x, gridDim.x), p.tiles_m, p.tiles_n, 1, tm, tn);
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

  const int64_t rbase = m0 + wr * G::WTM, cbase = n0 + wc * G::WTN;
  stage_barrier<0>();
  const Slab<G::WTN> s = {slab_of<G>(wave, lA0, lA1, lA2, lB0, lB1, lB2, lB3)};
  constexpr int LPR = G::WTN / 8;
  const int64_t c = cbase + (lane % LPR) * 8;
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = g.bias && c + e < g.N ? g.bias[c + e] : 0.f;
#pragma unroll
  for (int i = 0; i < G::TM; ++i) {
    slab_fill<G>(s, acc[i], [](int j) { return 32 * j; });
    // The adapters of these 32 rows, one after the other, in accumulators of
    // their own: carried round this loop, the tile's own would be copied out of
    // the accumulation registers and back (256 x 256: 96 registers spilled, and
    // operand pointers among them). A lane holds one row, and adds to it what
    // its own adapter gave: zeros for the other rows' T would not keep an
    // infinity or NaN of one request's adapter out of another's rows.
    const int64_t trow = rbase + 32 * i + (lane & 31);
    const int mine = adapter_of(g, trow);
    for (uint64_t todo = __ballot(mine >= 0); todo != 0;) {
      const int ad = __builtin_amdgcn_readlane(mine, __builtin_ctzll(todo));
      todo &= ~__ballot(mine == ad);
      const uint16_t* up = g.up + ad * g.stride_up;
      const uint16_t* tt = static_cast<const uint16_t*>(g.T) + trow * g.ldt;
      f32x16 own[G::TN];
#pragma unroll
      for (int j = 0; j < G::TN; ++j) own[j] = f32x16{};
#pragma unroll 1
      for (int r = 8 * (lane >> 5); r < g.ldt; r += 16) {
        // (a column past N re-reads the last one: its sums go nowhere)
        u32x4 b[G::TN];
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
          b[j] = load_row(up + min(cbase + 32 * j + (lane & 31), g.N - 1) * g.ld_up, r, g.R);
        const u32x4 v = mine == ad ? *reinterpret_cast<const u32x4*>(tt + r) : u32x4{};
#pragma unroll
        for (int j = 0; j < G::TN; ++j) own[j] = mfma32(b[j], v, own[j]);
      }
      if (mine == ad) {
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            s.add(lane & 31, 8 * j + 2 * q + (lane >> 5),
                  f32x4{own[j][4 * q], own[j][4 * q + 1], own[j][4 * q + 2], own[j][4 * q + 3]});
      }
    }
#pragma unroll 2
    for (int r = lane / LPR; r < 32; r += 64 / LPR) {
      const int64_t row = rbase + 32 * i + r;
      float v[8];
      s.get(r, lane % LPR, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bias[e];
      if (row >= g.M || c >= g.N) continue;
      if constexpr (OUT16)
        put8(static_cast<uint16_t*>(g.Y) + row * g.ldy, c, g.N, pack8(v));
      else
        put8f(static_cast<float*>(g.Y) + row * g.ldy, c, g.N, v);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A thread per column of one row (blockIdx.y).
template <bool OUT16>
__global__ __launch_bounds__(256) void k_adapter_sum(MultiArgs a, AdapterArgs g) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= g.N) return;
  const MultiProd& p = a.p[0];
  for (int64_t row = blockIdx.y; row < g.M; row += gridDim.y) {
    const int ad = __builtin_amdgcn_readfirstlane(adapter_of(g, row));
    const float* src = p.part + row * p.ldp + c;
    const int64_t slice = p.M * p.ldp;
    float v = src[0];
#pragma unroll 4
    for (int i = 1; i < a.pk; ++i) v += src[i * slice];
    if (g.bias) v += g.bias[c];
    if (ad >= 0) {
      const uint16_t* up = g.up + ad * g.stride_up + c * g.ld_up;
      const float* t = static_cast<const float*>(g.T) + row * g.ldt;
      for (int r = 0; r < g.R; r += 8) {
        float u[8];
        values8(get8(up, r, g.R), u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v += t[r + e] * u[e];  // (T holds zeros up to a multiple of 16)
      }
    }
    if constexpr (OUT16)
      static_cast<uint16_t*>(g.Y)[row * g.ldy + c] = to16(v);
    else
      static_cast<float*>(g.Y)[row * g.ldy + c] = v;
  }
}

template <int BM, int BN, int BK, int S>
hipError_t launch_tile(const MultiArgs& a, const AdapterArgs& g, int lay, bool out16, hipStream_t st) {
  const dim3 grid(a.p[0].tiles_m * a.p[0].tiles_n), block(256);
  if (lay == 0 && out16)
    hipLaunchKernelGGL((k_adapter<BM, BN, BK, S, 0, true>), grid, block, 0, st, a, g);
  else if (lay == 0)
    hipLaunchKernelGGL((k_adapter<BM, BN, BK, S, 0, false>), grid, block, 0, st, a, g);
  else if (out16)
    hipLaunchKernelGGL((k_adapter<BM, BN, BK, S, 2, true>), grid, block, 0, st, a, g);
  else
    hipLaunchKernelGGL((k_adapter<BM, BN, BK, S, 2, false>), grid, block, 0, st, a, g);
  return hipGetLastError();
}

}  // namespace

hipError_t adapter_shrink(const AdapterArgs& g, bool t16, hipStream_t st) {
  // 64 rows a workgroup where that leaves one for every CU
  const bool big = g.M >= 64 * 256;
  const int rows = big ? 64 : 16;
  const int64_t tiles = (g.M + rows - 1) / rows;
  if (tiles * rows >= (1LL << 31) / (64 * SW) || g.R < 1) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(tiles * rows), (unsigned)((g.R + 15) / 16)), block(64 * SW);
  if (t16 && big)
    hipLaunchKernelGGL((k_shrink<4, true>), grid, block, 0, st, g);
  else if (t16)
    hipLaunchKernelGGL((k_shrink<1, true>), grid, block, 0, st, g);
  else if (big)
    hipLaunchKernelGGL((k_shrink<4, false>), grid, block, 0, st, g);
  else
    hipLaunchKernelGGL((k_shrink<1, false>), grid, block, 0, st, g);
  return hipGetLastError();
}
hipError_t adapter_tile(const FfnTile& t, const MultiArgs& a, const AdapterArgs& g, int lay, bool out16,
                        hipStream_t st) {
  if (t.bm == 256 && t.bn == 256) return launch_tile<256, 256, 64, 2>(a, g, lay, out16, st);
  if (t.bm == 128 && t.bn == 256) return launch_tile<128, 256, 64, 3>(a, g, lay, out16, st);
  if (t.bm == 128 && t.bn == 128) return launch_tile<128, 128, 64, 2>(a, g, lay, out16, st);
  return hipErrorInvalidValue;
}
hipError_t adapter_sum(const MultiArgs& a, const AdapterArgs& g, bool out16, hipStream_t st) {
  const dim3 grid((unsigned)((g.N + 255) / 256), (unsigned)(g.M < 32768 ? g.M : 32768)), block(256);
  if (out16)
    hipLaunchKernelGGL((k_adapter_sum<true>), grid, block, 0, st, a, g);
  else
    hipLaunchKernelGGL((k_adapter_sum<false>), grid, block, 0, st, a, g);
  return hipGetLastError();
}

#if AC_INPUT_F16
}  // namespace f16
#endif
}  // namespace ac
