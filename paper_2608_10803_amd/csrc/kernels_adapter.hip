// gfx950 kernels of low-rank adapters beside a shared projection:
//   Y[i] = X[i] W + bias + T[i] up[a]^T,  T[i] = scale[a] X[i] down[a]^T,
//   a = index[i] (a row whose index is not one of the adapters has none),
// for rows of many requests in one product.
//
//   k_shrink       T, for every row. A workgroup takes 16 (or 64) rows, 16 of
//                  the rank and, in turn with the tile's other slots, the distinct
//                  adapters of those rows, which it finds itself, each for all
//                  the tile's rows of that adapter. So no sorting, no host
//                  knowledge of the indices, every adapter read once a tile, and
//                  all of a tile's adapters at once where there is a slot for
//                  each. K is split over the workgroup's waves.
//   k_multi_shrink few rows: the same beside the tiles of the shared product.
//   k_adapter      the shared product on the direct-to-LDS tile; before its
//                  epilogue each wave adds T up^T for the adapters of its rows,
//                  one after the other or (128 columns) four at a time, a row
//                  keeping what its own adapter gave, from global memory (R
//                  values a row and column against K of the main loop). Y is
//                  written once.
//   k_adapter_sum  few rows: adds the partial sums of the shared product,
//                  split along K, and T up^T by matrix instructions on two
//                  16-bit terms of T. There the adapters' bytes count like the
//                  weights': each is read where it is used once, R contiguous
//                  values a column.
//
// Measured, bf16, rank 16: 4096 rows of 8 requests on 4096 x 14336 k_shrink 16 us
// (its X at 2.1 TB/s: one workgroup a CU, two trips to memory after the index's)
// and k_adapter 454 us (1.06 PFLOP/s, bound by matrix instructions, 3.5 rounds of
// tiles); 16 rows of 16 adapters on 4096 x 4096 9.6 us for T and the partial sums
// (3.9 TB/s) and 5.1 for k_adapter_sum, bound by latency.
//
// Sums are fp32. k_adapter multiplies T by matrix instructions, so T is rounded
// to the input format there (one part in 2^9 of the adapters' share; in fp16 2^12,
// and past 65504 to infinity); k_adapter_sum, whose time is not the products',
// takes two terms (what is lost stands there).
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
  const int a = g.n > 0 && row < g.M ? g.index[row] : -1;  // (no adapters: index may be null)
  return a >= 0 && a < g.n ? a : -1;
}

// The distinct adapters of a tile's rows (lane: its row's adapter, `none` and
// below: not asked for), taken in turn by `slots` workgroups: the next one of
// slot `me`, with the rows that have it, or false at the end.
struct Groups {
  uint64_t todo;
  int turn;
  __device__ __forceinline__ void start(int mine, int none, int me) {
    todo = __ballot(mine > none);
    turn = me;
  }
  __device__ __forceinline__ bool next(int mine, int slots, int& a, uint64_t& rows) {
    while (todo != 0) {
      a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(todo));
      rows = __ballot(mine == a);
      todo &= ~rows;
      if (turn-- == 0) {
        turn = slots - 1;
        return true;
      }
    }
    return false;
  }
};

// T of MT * 16 rows (tile), 16 of the rank (rt), for the tile's adapters whose
// turn it is (me of slots). SW waves take 64 k each in turn. A lane loads 32
// contiguous bytes of a row, four lanes a line of it; the two halves go into
// two matrix instructions whose k are permuted alike in both operands. X's rows
// of other adapters are not loaded. U steps in flight; part: SW * MT * 256 floats.
template <int MT, int SW, bool T16>
__device__ __forceinline__ void shrink(const AdapterArgs& g, int tile, int me, int slots, int rt, float* part) {
  constexpr int ROWS = MT * 16, U = MT == 1 ? 4 : 1;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m0 = (int64_t)tile * ROWS;
  const int mine = lane < ROWS ? adapter_of(g, m0 + lane) : -1;
  const int r0 = rt * 16, i16 = lane & 15, kq = (lane >> 4) * 16;
  const uint16_t* x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x[m] = g.X + min(m0 + m * 16 + i16, g.M - 1) * g.ldx;
  const int64_t whole = g.K / 64;
  Groups of;
  of.start(mine, -1, me);
  int a;
  uint64_t rows;
  bool again = false;
  while (of.next(mine, slots, a, rows)) {
    const float scale = g.scale ? g.scale[a] : 1.0f;
    const uint16_t* down = g.down + a * g.stride_down + (int64_t)min(r0 + i16, g.R - 1) * g.ld_down;
    f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4{};
    // whole steps of 64 k, U of them in flight (zeros for those past the last: six
    // rows of 47 steps 10.4 us so, 11.9 with a loop of single steps after the last
    // whole batch), then the one that K ends in (not unrolled: its checked loads side
    // by side take more than the 128 registers there are)
    for (int64_t s = w; s < whole; s += U * SW) {
      u32x4 d[U][2], v[U][MT][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        d[u][0] = d[u][1] = u32x4{};
        if (u > 0 && s + u * SW >= whole) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) d[u][h] = load16(down + (s + u * SW) * 64 + kq + 8 * h);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u][m][0] = v[u][m][1] = u32x4{};
        if ((rows >> (m * 16 + i16)) & 1) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (u > 0 && s + u * SW >= whole) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) v[u][m][h] = load16(x[m] + (s + u * SW) * 64 + kq + 8 * h);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // every load on its way before the first product waits
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[m] = mfma16(v[u][m][h], d[u][h], acc[m]);
    }
    if (whole * 64 < g.K && whole % SW == w) {
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        const int64_t k = whole * 64 + kq + 8 * h;
        const u32x4 d = load_row(down, k, g.K);
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m] = mfma16(load_row(x[m], k, g.K), d, acc[m]);
      }
    }
    // the waves' sums, added in their order; lane: column i16, rows 4 * (lane >> 4) ..
    if (again) __syncthreads();  // the last adapter's have been read
    again = true;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[(w * MT + m) * 256 + ((lane >> 4) * 4 + e) * 16 + i16] = acc[m][e];
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * 16; i += 64 * SW) {
      const int row = i >> 4, r = r0 + (i & 15);
      if (!((rows >> row) & 1)) continue;
      float v = part[i];
#pragma unroll
      for (int j = 1; j < SW; ++j) v += part[j * MT * 256 + i];
      v = r < g.R ? v * scale : 0.f;
      if constexpr (T16)
        static_cast<uint16_t*>(g.T)[(m0 + row) * g.ldt + r] = to16(v);
      else
        static_cast<float*>(g.T)[(m0 + row) * g.ldt + r] = v;
    }
  }
}
// blockIdx.x: the row tile, blockIdx.y: the slot (with the slot running fastest
// the workgroups that have work, mostly the first slots', were all on one of
// the eight XCDs), blockIdx.z: 16 of the rank.
template <int MT, int SW, bool T16>
__global__ __launch_bounds__(64 * SW) __attribute__((amdgpu_waves_per_eu(4, 4))) void k_shrink(AdapterArgs g) {
  __shared__ float part[SW * MT * 256];
  shrink<MT, SW, T16>(g, blockIdx.x, blockIdx.y, gridDim.y, blockIdx.z, part);
}

// Few rows: T beside the partial sums of the shared product, in one launch
// (neither needs the other; as launches of their own 16 rows of 16 adapters on
// 4096 x 4096 take 10 and 8 us). The rows of the grid past the partitions do T:
// dispatched last, they share a CU with a tile each, where dispatched first they
// leave tiles to share one (32 rows of rank 32, 4096 x 14336: 44.4 us so, 39.5 now;
// other sizes within 3 %).
template <int BM, int BN, int BK, int S, int LAY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_multi_shrink(MultiArgs a, AdapterArgs g, int tiles, int slots) {
  typedef Dl<BM, BN, BK, S, LAY> G;
  typedef SegLoads<G> Loads;
  typedef FragAddrs<G> Addrs;
  constexpr bool RG = false;
  constexpr int OUT = DL_PARTIAL;
  AC_DL_STAGES(G);
  if ((int)blockIdx.y >= a.pk) {
    const int id = (blockIdx.y - a.pk) * gridDim.x + blockIdx.x, me = id / tiles % slots, rt = id / tiles / slots;
    static_assert(4 * 256 * 4 <= G::B_BYTES, "the waves' sums");
    if (rt * 16 < g.R) shrink<1, 4, false>(g, id % tiles, me, slots, rt, reinterpret_cast<float*>(lB0));
    return;
  }
  const int mblock = blockIdx.x, mblocks = gridDim.x;
#include "multi_tile.inc"
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
    // The adapters of these 32 rows. They go to accumulators of their own: carried
    // round their loop, the tile's own would be copied out of the accumulation
    // registers and back (256 x 256: 96 registers spilled, and operand pointers
    // among them). A lane holds one row, and keeps of each product what its own
    // adapter gave: zeros for the other rows' T would not keep an infinity or NaN
    // of one request's adapter out of another's rows.
    const int64_t trow = rbase + 32 * i + (lane & 31);
    const int mine = adapter_of(g, trow);
    if constexpr (G::TN > 2) {
      // one after the other, each added to the slab
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
    } else {
      // four at a time, their loads on their way together (1024 rows of as many
      // requests, 64 adapters of rank 16, 4096 x 4096: 112 us one after the other,
      // 87 so; on 256 x 256 the other way round, for 4096 rows of rank 64 900 and
      // 1058 us: its lanes hold twice the columns to choose from)
      constexpr int AT = 4;
      const uint64_t some = __ballot(mine >= 0);
      if (some != 0) {
        const uint16_t* tt = static_cast<const uint16_t*>(g.T) + trow * g.ldt;
        f32x16 sum[G::TN];
#pragma unroll
        for (int j = 0; j < G::TN; ++j) sum[j] = f32x16{};
#pragma unroll 1
        for (int r = 8 * (lane >> 5); r < g.ldt; r += 16) {
          const u32x4 v = mine >= 0 ? *reinterpret_cast<const u32x4*>(tt + r) : u32x4{};
#pragma unroll 1
          for (uint64_t todo = some; todo != 0;) {
            int ad[AT];
            u32x4 b[AT][G::TN];
#pragma unroll
            for (int q = 0; q < AT; ++q) {
              ad[q] = -2;
              if (todo != 0) {
                ad[q] = __builtin_amdgcn_readlane(mine, __builtin_ctzll(todo));
                todo &= ~__ballot(mine == ad[q]);
                // (a column past N re-reads the last one: its sums go nowhere)
                const uint16_t* up = g.up + ad[q] * g.stride_up;
#pragma unroll
                for (int j = 0; j < G::TN; ++j)
                  b[q][j] = load_row(up + min(cbase + 32 * j + (lane & 31), g.N - 1) * g.ld_up, r, g.R);
              }
            }
#pragma unroll
            for (int q = 0; q < AT; ++q) {
              if (ad[q] < 0) continue;
              const bool its = mine == ad[q];
#pragma unroll
              for (int j = 0; j < G::TN; ++j) {
                const f32x16 one = mfma32(b[q][j], its ? v : u32x4{}, sum[j]);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[j][e] = its ? one[e] : sum[j][e];
              }
            }
          }
        }
        if (mine >= 0) {
#pragma unroll
          for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              s.add(lane & 31, 8 * j + 2 * q + (lane >> 5),
                    f32x4{sum[j][4 * q], sum[j][4 * q + 1], sum[j][4 * q + 2], sum[j][4 * q + 3]});
        }
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

// A workgroup takes `per` rows of one adapter (or of the rows without) out of a
// tile of tile_rows <= 64 (blockIdx.y), wherever they lie in it, then those that
// are its slot's next (blockIdx.z), for 256 columns (blockIdx.x), 64 a wave. T
// up^T by matrix instructions for up to 16 rows at once: their operand takes up
// as it lies in memory, 16 columns of 32 consecutive values an instruction,
// where a lane that walks its column's R values touches 64 lines with every load
// (64 rows of 32 adapters of rank 64, 14336 columns: 34 us that way). T goes in
// as the sum of two 16-bit values, so what is lost of it is 2^-16 (bf16) of each
// value and less. fp16 has neither fp32's range nor its small values: there a
// row's T goes in times the power of two that brings its greatest finite value
// so far just below 2^15 (the sums follow when a later value is greater), and
// what is lost is 2^-22 of the row's greatest.
//
// per: 4 up to 256 rows, else 16. A prompt's rows are so spread over the slots
// (4096 x 4096, rank 16: 64 rows of 3 requests 29 us, 58 where a slot takes all
// rows of an adapter; 128 rows of 4 requests 30 and 44). What is left is the
// traffic of the partial sums, up and Y: 64 rows of 32 adapters of rank 64 on
// 14336 columns take 18 us (59 MB of up: 3.3 TB/s).
//
// R8: the rank is a multiple of 8 (no partial chunk of up), which takes few
// enough registers for four waves a SIMD.
template <bool OUT16, bool R8>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(R8 ? 4 : 3))) void k_adapter_sum(MultiArgs a,
                                                                                                    AdapterArgs g,
                                                                                                    int tile_rows,
                                                                                                    int per) {
  __shared__ float box[4][16][64 + 4];
  constexpr bool SCALED = AC_INPUT_F16 != 0;
  constexpr int NO_EX = -1000;  // of a row of zeros
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i16 = lane & 15;
  const int64_t mt = (int64_t)blockIdx.y * tile_rows;
  const int64_t c0 = (int64_t)blockIdx.x * 256 + w * 64;
  if (c0 >= g.N) return;  // (no barrier below: a wave reads only what it wrote)
  // for the partial sums and the stores: four rows at a time, 16 lanes a row,
  // four columns a lane
  const MultiProd& p = a.p[0];
  const int64_t slice = p.M * p.ldp;
  const int64_t c = c0 + i16 * 4;
  float bias[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) bias[e] = g.bias && c + e < g.N ? g.bias[c + e] : 0.f;
  const int mine = lane < tile_rows && mt + lane < g.M ? adapter_of(g, mt + lane) : -2;
  uint64_t left = __ballot(mine > -2);
  int turn = blockIdx.z;
  while (left != 0) {
    const int ad = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
    const uint64_t group = __ballot(mine == ad);
    left &= ~group;
    const int items = (__builtin_popcountll(group) + per - 1) / per;
#pragma unroll 1
    for (; turn < items; turn += gridDim.z) {
      uint64_t rest = group;
      for (int i = 0; i < turn * per; ++i) rest &= rest - 1;
      // the item's n rows; lane: the row of place i16 (0: none there)
      int n = 0, at = 0;
      for (; n < per && rest != 0; ++n, rest &= rest - 1) at = i16 == n ? __builtin_ctzll(rest) : at;
      // the four rows from place q on: the lane's of them, and its first four
      // partial sums (the last one again where there are fewer)
      int row;
      f32x4 s[4];
      auto fetch = [&](int from) {
#pragma unroll
        for (int h = 0; h < 4; ++h)
          s[h] = *reinterpret_cast<const f32x4*>(p.part + (mt + row) * p.ldp + min(c, p.ldp - 4) +
                                                 min(from + h, a.pk - 1) * slice);
      };
      auto rows_from = [&](int q) {
        row = __shfl(at, q + (lane >> 4));
        fetch(0);
      };
      rows_from(0);  // on their way while T up^T is made
      if (ad >= 0) {
        const int kq = (lane >> 4) * 8;
        f32x4 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = f32x4{};
        const uint16_t* up[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) up[j] = g.up + ad * g.stride_up + min(c0 + 16 * j + i16, g.N - 1) * g.ld_up;
        const float* tt = static_cast<const float*>(g.T) + (mt + at) * g.ldt;
        int ex = NO_EX;
        for (int r = 0; r < g.R; r += 32) {
          u32x4 b[4], hi, lo;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            b[j] = r + kq < g.R ? (R8 ? load16(up[j] + r + kq) : get8(up[j], r + kq, g.R)) : u32x4{};
          float t8[8] = {};
          if (i16 < n && r + kq < g.ldt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const f32x4 v = *reinterpret_cast<const f32x4*>(tt + r + kq + 4 * h);
#pragma unroll
              for (int e = 0; e < 4; ++e) t8[4 * h + e] = v[e];
            }
          }
          if constexpr (SCALED) {
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(t8[e]) < INFINITY ? fabsf(t8[e]) : 0.f);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const int now = max(ex, top > 0.f ? __builtin_amdgcn_frexp_expf(top) - 15 : NO_EX);
            if (__any(now > ex)) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int down = __shfl(ex - now, (lane >> 4) * 4 + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][e] = ldexpf(acc[j][e], down);
              }
            }
            ex = now;
#pragma unroll
            for (int e = 0; e < 8; ++e) t8[e] = ldexpf(t8[e], -ex);
          }
          float t0[8], t1[8];
          hi = pack8(t8);
          values8(hi, t0);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = t8[e] - t0[e];
            t1[e] = fabsf(d) < INFINITY ? d : 0.f;  // (an infinity stays one)
          }
          lo = pack8(t1);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = mfma16(lo, b[j], mfma16(hi, b[j], acc[j]));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row_ex = SCALED ? __shfl(ex, (lane >> 4) * 4 + e) : 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            box[w][(lane >> 4) * 4 + e][16 * j + i16] = SCALED ? ldexpf(acc[j][e], row_ex) : acc[j][e];
        }
      }
#pragma unroll 1
      for (int q = 0; q < n; q += 4) {
        f32x4 v = s[0];
#pragma unroll
        for (int h = 1; h < 4; ++h)
          if (h < a.pk) v += s[h];
        for (int f = 4; f < a.pk; f += 4) {
          fetch(f);
#pragma unroll
          for (int h = 0; h < 4; ++h)
            if (f + h < a.pk) v += s[h];
        }
        const int place = q + (lane >> 4);
        const int64_t m = mt + row;
        if (q + 4 < n) rows_from(q + 4);
        if (place >= n || c >= g.N) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += bias[e];
        if (ad >= 0) v += *reinterpret_cast<const f32x4*>(&box[w][place][i16 * 4]);
        if constexpr (OUT16) {
          uint16_t* y = static_cast<uint16_t*>(g.Y) + m * g.ldy;
          if (c + 4 <= g.N) {
            const uint64_t bits = (uint64_t)to16(v[0]) | ((uint64_t)to16(v[1]) << 16) | ((uint64_t)to16(v[2]) << 32) |
                                  ((uint64_t)to16(v[3]) << 48);
            __builtin_memcpy(y + c, &bits, 8);
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (c + e < g.N) y[c + e] = to16(v[e]);
          }
        } else {
          float* y = static_cast<float*>(g.Y) + m * g.ldy;
          if (c + 4 <= g.N) {
            __builtin_memcpy(y + c, &v, 16);
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (c + e < g.N) y[c + e] = v[e];
          }
        }
      }
    }
    turn -= items;
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

// Slots of a row tile of 16: enough workgroups for twice the CUs where the rows
// are few, each of whose rows may have its own adapter; a prompt's tiles have one
// or two, and workgroups without work cost as much as the others' start (4096
// rows of 8 requests: 18 us with one slot, 21 with two, 23 with four).
static int slots_of(int64_t tiles) { return (int)(tiles >= 256 ? 1 : tiles <= 32 ? 16 : 512 / tiles); }

hipError_t adapter_shrink(const AdapterArgs& g, bool t16, hipStream_t st) {
  if (g.R < 1 || g.R > 4096) return hipErrorInvalidValue;
  const int rt = (g.R + 15) / 16;
  if (g.M >= 64 * 256) {  // 64 rows a workgroup leave one for every CU
    const dim3 grid((unsigned)((g.M + 63) / 64), 1, rt), block(512);
    if (t16)
      hipLaunchKernelGGL((k_shrink<4, 8, true>), grid, block, 0, st, g);
    else
      hipLaunchKernelGGL((k_shrink<4, 8, false>), grid, block, 0, st, g);
  } else {
    const int64_t tiles = (g.M + 15) / 16;
    const dim3 grid((unsigned)tiles, slots_of(tiles), rt), block(512);
    if (t16)
      hipLaunchKernelGGL((k_shrink<1, 8, true>), grid, block, 0, st, g);
    else
      hipLaunchKernelGGL((k_shrink<1, 8, false>), grid, block, 0, st, g);
  }
  return hipGetLastError();
}
hipError_t adapter_multi_shrink(const MultiArgs& a, const AdapterArgs& g, int lay, hipStream_t st) {
  const int tiles = (int)((g.M + 15) / 16), rt = (g.R + 15) / 16, slots = slots_of(tiles);
  if (g.M > 64 || g.R < 1 || g.R > 4096 || a.n != 1 || a.pk < 1) return hipErrorInvalidValue;
  const int wide = a.p[0].tiles_m * a.p[0].tiles_n;
  const dim3 grid(wide, a.pk + (tiles * slots * rt + wide - 1) / wide), block(256);
  if (lay == 0)
    hipLaunchKernelGGL((k_multi_shrink<32, 128, 64, 4, 0>), grid, block, 0, st, a, g, tiles, slots);
  else
    hipLaunchKernelGGL((k_multi_shrink<32, 128, 64, 4, 2>), grid, block, 0, st, a, g, tiles, slots);
  return hipGetLastError();
}
hipError_t adapter_tile(const FfnTile& t, const MultiArgs& a, const AdapterArgs& g, int lay, bool out16,
                        hipStream_t st) {
  if (t.bm != t.bn) return hipErrorInvalidValue;
  if (t.bm == 256 && t.stages == 2) return launch_tile<256, 256, 64, 2>(a, g, lay, out16, st);
  if (t.bm == 128 && t.stages == 2) return launch_tile<128, 128, 64, 2>(a, g, lay, out16, st);
  if (t.bm == 128 && t.stages == 3) return launch_tile<128, 128, 64, 3>(a, g, lay, out16, st);
  return hipErrorInvalidValue;
}
// (row tiles beyond what one launch's grid takes in launches of their own)
hipError_t adapter_sum(const MultiArgs& a, const AdapterArgs& g, bool out16, hipStream_t st) {
  const int rows = g.M > 16 ? 64 : 16;  // of a tile
  const int64_t most = (int64_t)65535 * rows;
  for (int64_t m = 0; m < g.M; m += most) {
    MultiArgs a2 = a;
    AdapterArgs g2 = g;
    g2.M = g.M - m < most ? g.M - m : most;
    if (g.index != nullptr) g2.index += m;
    a2.p[0].part += m * a.p[0].ldp;  // (a slice is still p.M rows)
    g2.T = g.T == nullptr ? nullptr : static_cast<float*>(g.T) + m * g.ldt;
    g2.Y = static_cast<char*>(g.Y) + m * g.ldy * (out16 ? 2 : 4);
    const int64_t tiles = (g2.M + rows - 1) / rows, chunks = (g.N + 255) / 256;
    const int slots = rows == 16 ? 16 : (int)(tiles <= 8 ? 32 : tiles >= 256 ? 1 : 256 / tiles);
    const int per = tiles <= 4 ? 4 : 16;
    const dim3 grid((unsigned)chunks, (unsigned)tiles, slots), block(256);
#define AC_SUM(O, R8)                        \
  if (out16 == O && (g.R % 8 == 0) == R8)    \
    hipLaunchKernelGGL((k_adapter_sum<O, R8>), grid, block, 0, st, a2, g2, rows, per);
    AC_SUM(true, true)
    AC_SUM(true, false)
    AC_SUM(false, true)
    AC_SUM(false, false)
#undef AC_SUM
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

#if AC_INPUT_F16
}  // namespace f16
#endif
}  // namespace ac
