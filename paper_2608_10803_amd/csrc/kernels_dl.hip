// gfx950 macro-tile kernels whose operand tiles travel from global memory
// straight into LDS (buffer_load ... lds: no staging registers, no register
// transposes) through S LDS stages, so that S - 1 k-blocks of loads are in
// flight while one is multiplied out (the Multi-Buffer module of Table 2;
// the schedule of Eq. 13 with a deeper pipeline).
//
//   A tile  BM x 64 k, row-major as in memory, 16-byte chunks XOR-swizzled
//           per row; MFMA fragments read with ds_read_b128.
//   B tile  64 k x BN, row-major as in memory (chunks swizzled per k-row);
//           MFMA fragments read with the LDS transpose read
//           ds_read_b64_tr_b16, which hands each lane four consecutive k of
//           one column: the k-contiguous operand the MFMA needs, without the
//           v_perm transposes of the register-staged kernel.
//   C       4 waves in a 2 x 2 grid, each a (BM/2) x (BN/2) quadrant of
//           32 x 32 x 16 MFMAs (tiles of at most 64 rows: 4 waves side by
//           side along N); fp32 accumulation in the accumulation registers;
//           bf16 output converted through a per-wave LDS slab and written as
//           whole 16-byte row segments.
//
// The swizzle of a stage is applied on the global side: a wave-wide LDS load
// writes 1024 contiguous bytes (lane l to bytes 16l .. 16l+15), so each lane
// fetches the global chunk that belongs at its slot.
//
// (A column-major operand read in place, k_dlc, trades places: a B of N rows
// of k is tiled and read like A here, an A of K rows of M like B.)
//
// k_dl needs row-major operands with 16-byte aligned rows (A and B base
// addresses 16-byte aligned, lda and ldb multiples of 8 below 2^22) and K, N
// multiples of 8. A plan for other shapes either copies the operand
// zero-padded first (k_pad16 below, the Padding module) or runs k_dlu, the
// register-load form of the same tiling (16-byte loads at any 2-byte
// alignment, two LDS stages); an operand found misaligned at run time takes
// k_dlu, or the register-staged tile kernel of the same tiling where the
// configuration has no k_dlu. Chunks outside the matrices (rows past M,
// columns past N, k past K) are read as zeros through out-of-range buffer
// offsets, so edge tiles take the same path.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernel_args.h"
#include "registry.h"

#ifndef AC_INPUT_F16
#define AC_INPUT_F16 0
#endif
#ifndef AC_DL_PART
#define AC_DL_PART 0
#endif

namespace ac {
#if AC_INPUT_F16
namespace f16 {
#endif

#include "device_common.h"
#include "grouped_map.h"

namespace {

#include "dl_pipeline.h"

// One output tile (tile coordinates tm, tn) over K partition `split` of the
// plan's kper-block partitions.
template <int BM, int BN, int BK, int S, int OUT, bool RG, int LAY = 0>
__device__ __forceinline__ void dl_tile(const GemmArgs& g, int tm, int tn, int split) {
  typedef Dl<BM, BN, BK, S, LAY> G;
  typedef typename std::conditional<RG, DlTileU<G>, DlTile<G>>::type Tile;
  typedef typename std::conditional<RG, RegLoads<G>, StageLoads<G>>::type Loads;
  typedef FragAddrs<G> Addrs;
  AC_DL_STAGES(G);
  static_assert(S >= 2 && S <= 5, "stages");

  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  // the K partition: kper blocks of the plan's 64-deep granule, a whole
  // number of this kernel's k-blocks
  const int64_t kbeg = min((int64_t)split * g.kper * 64, g.K);
  const int64_t kend = min(kbeg + (int64_t)g.kper * 64, g.K);
  const int nk = (int)((kend - kbeg + G::BK - 1) / G::BK);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave / G::WN, wc = wave % G::WN;

  Tile t;
  t.init(g, m0, n0);

#include "dl_main_loop.inc"

  // ---- epilogue
  const int64_t rbase = m0 + wr * G::WTM, cbase = n0 + wc * G::WTN;
  if constexpr (OUT == DL_BF16) {
    stage_barrier<0>();  // every wave's last reads of the stages are done, no load into them is in flight
    // the wave's slab: 32 rows x WTN bf16 in one of the stage buffers
    char* slab;
    if constexpr (G::SLAB_KIND == 0)
      slab = wave == 0 ? lA0 : wave == 1 ? lA1 : wave == 2 ? lB0 : lB1;
    else if constexpr (G::SLAB_KIND == 1)
      slab = wave == 0 ? lB0 : wave == 1 ? lB1 : wave == 2 ? lB2 : lB3;
    else if constexpr (G::SLAB_KIND == 3)
      slab = (wave < 2 ? lB0 : lB1) + (wave & 1) * G::SLAB;
    else
      slab = wave == 0 ? lA0 : wave == 1 ? lA1 : wave == 2 ? lA2 : lA3;
    uint16_t* ct = reinterpret_cast<uint16_t*>(slab);
    uint16_t* C = static_cast<uint16_t*>(g.C);
    constexpr int GPR = G::WTN / 8;  // 16-byte groups per slab row
#pragma unroll
    for (int i = 0; i < G::TM; ++i) {
      const int64_t row = rbase + 32 * i + (lane & 31);
#pragma unroll
      for (int j = 0; j < G::TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = 32 * j + (q << 3) + ((lane >> 5) << 2);  // acc elements 4q .. 4q+3: four columns
          float w[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          if (g.epi && row < g.M && cbase + c < g.N) epi_apply<true, 4>(g, w, row, cbase + c, g.N - cbase - c);
          const uint32_t lo = (uint32_t)to16(w[0]) | ((uint32_t)to16(w[1]) << 16);
          const uint32_t hi = (uint32_t)to16(w[2]) | ((uint32_t)to16(w[3]) << 16);
          *reinterpret_cast<uint64_t*>(ct + (lane & 31) * G::CT_LD + c) = (uint64_t)lo | ((uint64_t)hi << 32);
        }
      // the slab back as 16-byte row segments (the same wave: LDS is in order)
#pragma unroll
      for (int v = 0; v < 32 * GPR / 64; ++v) {
        const int u = lane + 64 * v, r = u / GPR, grp = u % GPR;
        const uint16_t* src = ct + r * G::CT_LD + grp * 8;
        const uint64_t a = *reinterpret_cast<const uint64_t*>(src);
        const uint64_t b = *reinterpret_cast<const uint64_t*>(src + 4);
        const int64_t gr = rbase + 32 * i + r, gc = cbase + grp * 8;
        if (gr < g.M && gc + 8 <= g.N) {
          const uint64_t vv[2] = {a, b};
          __builtin_memcpy(C + gr * g.ldc + gc, vv, 16);
        } else if (gr < g.M && gc < g.N) {  // the last, partial group of a row
          const uint16_t* e = src;
          for (int j = 0; j < (int)(g.N - gc); ++j) C[gr * g.ldc + gc + j] = e[j];
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // slab by slab: bounded live registers
    }
  } else {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // no load into LDS outlives the workgroup
    float* dst = OUT == DL_PARTIAL ? g.ws + (size_t)split * (size_t)g.M * (size_t)g.ldw : static_cast<float*>(g.C);
    const int64_t ld = OUT == DL_PARTIAL ? g.ldw : g.ldc;
#pragma unroll
    for (int i = 0; i < G::TM; ++i) {
      const int64_t row = rbase + 32 * i + (lane & 31);
      if (row >= g.M) continue;
#pragma unroll
      for (int j = 0; j < G::TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t col = cbase + 32 * j + (q << 3) + ((lane >> 5) << 2);
          if (col >= g.N) continue;
          float w[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          if (OUT == DL_F32 && g.epi) epi_apply<false, 4>(g, w, row, col, g.N - col);
          if (col + 4 <= g.N) {
            const f32x4 vv = {w[0], w[1], w[2], w[3]};
            __builtin_memcpy(dst + row * ld + col, &vv, 16);
          } else {
            for (int e = 0; e < (int)(g.N - col); ++e) dst[row * ld + col + e] = w[e];
          }
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// a workgroup per output tile (blockIdx.x, in the plan's tile order) and K
// partition (blockIdx.y)
template <int BM, int BN, int BK, int S, int OUT, bool RG, int LAY = 0>
__device__ __forceinline__ void dl_kernel(const GemmArgs& g) {
  const int ntiles = g.tiles_m * g.tiles_n;
  int tile = blockIdx.x;
  if (g.swizzle) tile = xcd_remap(tile, ntiles);
  int tm, tn;
  tile_coords(tile, g.tiles_m, g.tiles_n, g.swizzle, tm, tn);
  // the division ran in vector registers: back to scalar ones, or the
  // operand pointers stay there and every load loops over its lanes' pointers
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  dl_tile<BM, BN, BK, S, OUT, RG, LAY>(g, tm, tn, (int)blockIdx.y);
}

// the kernels: operand tiles loaded straight into LDS (k_dl), or through
// registers at any alignment (k_dlu)
template <int BM, int BN, int BK, int S, int OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_dl(GemmArgs g) {
  dl_kernel<BM, BN, BK, S, OUT, false>(g);
}
template <int BM, int BN, int BK, int S, int OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_dlu(GemmArgs g) {
  dl_kernel<BM, BN, BK, S, OUT, true>(g);
}

// the same with one operand column-major in memory, read in place (LAY 1: A,
// LAY 2: B): no transposed copy, the same bits
template <int BM, int BN, int BK, int S, int OUT, int LAY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_dlc(GemmArgs g) {
  dl_kernel<BM, BN, BK, S, OUT, false, LAY>(g);
}

// Off-chip accumulation (the SingleCoreSplitK and HybridSplitK templates of
// Section 4.2; write volume of Eqs. 3 and 5): a workgroup owns a super-tile
// of two vertically adjacent tiles, 2BM x BN, whose fp32 accumulator does not
// fit the registers, and takes the plan's P_k k1-slices of K in order --
// all of them (gridDim.y = 1: SingleCoreSplitK) or its share of them
// (gridDim.y workgroups along K: HybridSplitK). For every slice it computes
// the upper tile, flushes its partial sums to the slice's fp32 partial buffer
// in the workspace, then the lower tile (whose B slice the upper one has just
// brought into the L2); the reduction kernel then adds the slices. Each tile
// of each slice is the direct-to-LDS tile kernel's own computation of that
// partition, so the result has the bits of the split-K plan with the same
// partitions.
template <int BM, int BN, int BK, int S>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_dl_sc(GemmArgs g) {
  const int sup = blockIdx.x;
  const int stm = __builtin_amdgcn_readfirstlane(sup / g.tiles_n), tn = sup - stm * g.tiles_n;
  const int per = g.pk / (int)gridDim.y;  // slices of this workgroup
  for (int q = 0; q < per; ++q) {
    const int split = (int)blockIdx.y * per + q;
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      const int tm = 2 * stm + h;
      if (tm >= g.tiles_m) break;
      // the previous tile's loads and stores are complete and no wave still
      // reads its LDS stages
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __syncthreads();
      dl_tile<BM, BN, BK, S, DL_PARTIAL, false>(g, tm, tn, split);
    }
  }
}

// The grouped and strided-batch products on the direct-to-LDS tile (one tile
// of one group per workgroup, no K split): k_grouped's tiles and the same
// sums, so its bits, on operands whose every group has aligned rows.
//
// Tile order of a grouped product (swizzle): the tiles of a group run column
// panel by column panel, its row tiles one after the other (they share the
// panel's B), and the XCDs take GRP_CHUNK consecutive tiles in turn. Giving
// each XCD one contiguous eighth of the tiles, as for a plain product, left
// some XCDs with the heavy groups, whose tiles share B in the L2, and others
// with the light ones, each of whose tiles streams a panel of its own from
// HBM. 8192 rows over 64 groups of unequal load, K 4096, N 1536, 128 x 256
// tiles: register-staged 290 us, this kernel in that order 233, in chunks of
// one tile 242, 2: 221, 4: 214, 8: 209, 12: 212. On 30 products of 4 to 64
// groups (64-8192 rows, N and K 256-4096), chunks of 1, 4 and 16 take 1.118x,
// 1.019x and 1.016x the time of 8 in the geometric mean.
constexpr int GRP_CHUNK = 8;

template <int BM, int BN, int BK, int S, int OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Dl<BM, BN, BK, S>::WPE, Dl<BM, BN, BK, S>::WPE)))
void k_grouped_dl(GroupArgs a) {
  const int tiles_n = a.g.tiles_n;
  int t = blockIdx.x;
  int grp = 0, tm = 0, tn = 0;
  int64_t row0 = 0, rows_g = 0;
  if (a.counts == nullptr) {
    // strided batch: the grid is exactly groups x row tiles x column tiles
    if (a.g.swizzle) t = xcd_remap(t, (int)gridDim.x);
    const int slot = t / tiles_n;
    tn = t - slot * tiles_n;
    grp = slot / a.tiles_per_group;
    tm = slot - grp * a.tiles_per_group;
    rows_g = a.rows;
  } else {
    GroupChunk<BM> first;
    first.load(a, 0, 0);
    if (a.g.swizzle) {
      // over the tiles that exist: whole rounds of 8 chunks, the rest in order
      const int n = group_tiles_total<BM>(a, first) * tiles_n;
      if (t >= n) return;
      const int whole = n / (8 * GRP_CHUNK) * (8 * GRP_CHUNK);
      if (t < whole) {
        const int i = t >> 3;
        t = (i / GRP_CHUNK) * (8 * GRP_CHUNK) + (t & 7) * GRP_CHUNK + i % GRP_CHUNK;
      }
    }
    const int slot = t / tiles_n;
    if (!group_of_slot<BM>(a, first, slot, grp, row0, rows_g, tm)) return;
    // the group's tiles start at its first slot's
    const int in = t - (slot - tm) * tiles_n, rt = (int)((rows_g + BM - 1) / BM);
    tn = in / rt;
    tm = in - tn * rt;
  }
  // the same values in every lane: scalar for the address bases
  grp = __builtin_amdgcn_readfirstlane(grp);
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  row0 = uniform64(row0);
  rows_g = uniform64(rows_g);

  GemmArgs g = a.g;
  g.A += row0 * g.lda + (int64_t)grp * a.stride_a;
  g.B += (int64_t)grp * a.stride_b;
  g.C = static_cast<char*>(g.C) + (row0 * g.ldc + (int64_t)grp * a.stride_c) * (OUT == DL_BF16 ? 2 : 4);
  if (g.epi && g.bias != nullptr) g.bias += (int64_t)grp * a.stride_bias;
  g.M = rows_g;
  dl_tile<BM, BN, BK, S, OUT, false>(g, tm, tn, 0);
}

template <int BM, int BN, int BK, int S, int OUT>
void start_dl(const GemmArgs& g, dim3 grid, hipStream_t st) {
  const dim3 block(256);
  if constexpr ((dl_col(BM, BN, BK, S) & 1) != 0)
    if (g.lay == 1) {
      hipLaunchKernelGGL((k_dlc<BM, BN, BK, S, OUT, 1>), grid, block, 0, st, g);
      return;
    }
  if constexpr ((dl_col(BM, BN, BK, S) & 2) != 0)
    if (g.lay == 2) {
      hipLaunchKernelGGL((k_dlc<BM, BN, BK, S, OUT, 2>), grid, block, 0, st, g);
      return;
    }
  hipLaunchKernelGGL((k_dl<BM, BN, BK, S, OUT>), grid, block, 0, st, g);
}

}  // namespace

// The launcher and the occupancy of one configuration. A configuration's
// kernels are compiled where these are instantiated: the file is compiled
// once per AC_DL_PART, each part with its configurations, so that the build
// runs in parallel.
template <int BM, int BN, int BK, int S>
hipError_t launch_dl(const Plan& p, const GemmArgs& g, hipStream_t st, bool obf) {
  const dim3 grid(p.grid_x, p.grid_y), block(256);
  if (g.lay != 0 && (p.unal || g.lay == 3 || (g.lay & ~dl_col(BM, BN, BK, S)) != 0)) return hipErrorInvalidValue;
  if (p.unal) {
    if constexpr (dl_has_unal(BM, BN, BK, S)) {
      if (p.pk > 1)
        hipLaunchKernelGGL((k_dlu<BM, BN, BK, S, DL_PARTIAL>), grid, block, 0, st, g);
      else if (obf)
        hipLaunchKernelGGL((k_dlu<BM, BN, BK, S, DL_BF16>), grid, block, 0, st, g);
      else
        hipLaunchKernelGGL((k_dlu<BM, BN, BK, S, DL_F32>), grid, block, 0, st, g);
    } else {
      return hipErrorInvalidValue;
    }
  } else if (p.pk > 1) {
    start_dl<BM, BN, BK, S, DL_PARTIAL>(g, grid, st);
  } else if (obf) {
    start_dl<BM, BN, BK, S, DL_BF16>(g, grid, st);
  } else {
    start_dl<BM, BN, BK, S, DL_F32>(g, grid, st);
  }
  return hipGetLastError();
}

// Workgroups per CU for the planner: the device's figure, but no more than
// the configuration is built for, which is what its costs were fitted with
// (28921 x 20011 x 59: a 128 x 128 x 32 tile priced at three per CU was taken
// at 320 us where the 64 x 512 one runs in 298).
template <int BM, int BN, int BK, int S>
int occ_dl() {
  int o = Dl<BM, BN, BK, S>::WPE;
  const void* ks[6] = {reinterpret_cast<const void*>(k_dl<BM, BN, BK, S, DL_F32>),
                       reinterpret_cast<const void*>(k_dl<BM, BN, BK, S, DL_BF16>),
                       reinterpret_cast<const void*>(k_dl<BM, BN, BK, S, DL_PARTIAL>), nullptr, nullptr, nullptr};
  if constexpr (dl_has_unal(BM, BN, BK, S)) {  // the register-load form: one occupancy for both
    ks[3] = reinterpret_cast<const void*>(k_dlu<BM, BN, BK, S, DL_F32>);
    ks[4] = reinterpret_cast<const void*>(k_dlu<BM, BN, BK, S, DL_BF16>);
    ks[5] = reinterpret_cast<const void*>(k_dlu<BM, BN, BK, S, DL_PARTIAL>);
  }
  for (const void* k : ks) {
    if (!k) continue;
    int a = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&a, k, 256, 0) != hipSuccess) a = 0;
    o = a < o ? a : o;
  }
  return o;
}

template <int BM, int BN, int BK, int S>
hipError_t launch_grouped_dl(const Plan& p, const GroupArgs& a, hipStream_t st, bool obf) {
  const dim3 grid(p.grid_x), block(256);
  if (obf)
    hipLaunchKernelGGL((k_grouped_dl<BM, BN, BK, S, DL_BF16>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_grouped_dl<BM, BN, BK, S, DL_F32>), grid, block, 0, st, a);
  return hipGetLastError();
}
#define GDL_INST(a, b, c, d) template hipError_t launch_grouped_dl<a, b, c, d>(const Plan&, const GroupArgs&, hipStream_t, bool);
#define GDL_EXT(a, b, c, d) extern GDL_INST(a, b, c, d)
#define DL_INST(a, b, c, d)                                                                   \
  template hipError_t launch_dl<a, b, c, d>(const Plan&, const GemmArgs&, hipStream_t, bool); \
  template int occ_dl<a, b, c, d>();
#define DL_EXT(a, b, c, d)                                                                           \
  extern template hipError_t launch_dl<a, b, c, d>(const Plan&, const GemmArgs&, hipStream_t, bool); \
  extern template int occ_dl<a, b, c, d>();
// (a configuration is in one part; the static assertion on DL_CFGS below and
// the linker hold the parts and the table together)
#if AC_DL_PART == 1
DL_INST(256, 256, 64, 2)
#elif AC_DL_PART == 2
DL_INST(256, 256, 32, 4)
DL_INST(256, 256, 32, 5)
#elif AC_DL_PART == 3
DL_INST(256, 128, 64, 3)
DL_INST(128, 256, 64, 3)
#elif AC_DL_PART == 4
DL_INST(256, 128, 32, 4)
DL_INST(128, 256, 32, 4)
DL_INST(128, 128, 64, 3)
#elif AC_DL_PART == 5
DL_INST(256, 128, 32, 2)
DL_INST(128, 128, 64, 2)
DL_INST(128, 128, 32, 2)
#elif AC_DL_PART == 6
DL_INST(32, 256, 64, 4)
DL_INST(64, 256, 64, 4)
DL_INST(32, 128, 64, 4)
DL_INST(64, 512, 32, 2)
#elif AC_DL_PART == 7
GDL_INST(256, 128, 64, 3)
GDL_INST(128, 256, 64, 3)
GDL_INST(128, 128, 64, 2)
GDL_INST(128, 128, 64, 3)
GDL_INST(64, 128, 64, 3)
#else
GDL_EXT(256, 128, 64, 3) GDL_EXT(128, 256, 64, 3) GDL_EXT(128, 128, 64, 2) GDL_EXT(128, 128, 64, 3)
GDL_EXT(64, 128, 64, 3)
DL_EXT(256, 256, 64, 2) DL_EXT(256, 256, 32, 4) DL_EXT(256, 256, 32, 5) DL_EXT(256, 128, 64, 3)
DL_EXT(128, 256, 64, 3) DL_EXT(256, 128, 32, 4) DL_EXT(128, 256, 32, 4) DL_EXT(128, 128, 64, 3)
DL_EXT(256, 128, 32, 2) DL_EXT(128, 128, 64, 2) DL_EXT(128, 128, 32, 2) DL_EXT(32, 256, 64, 4)
DL_EXT(64, 256, 64, 4) DL_EXT(32, 128, 64, 4) DL_EXT(64, 512, 32, 2)

namespace {
typedef hipError_t (*DlLaunchFn)(const Plan&, const GemmArgs&, hipStream_t, bool);
typedef int (*DlOccFn)();
#define DL_CFGS(X) X(256, 256, 64, 2), X(256, 128, 64, 3), X(128, 256, 64, 3), X(128, 128, 64, 3), X(256, 256, 32, 4), \
    X(256, 256, 32, 5), X(256, 128, 32, 4), X(128, 256, 32, 4), X(256, 128, 32, 2), X(128, 128, 64, 2),       \
    X(128, 128, 32, 2), X(32, 256, 64, 4), X(64, 256, 64, 4), X(32, 128, 64, 4), X(64, 512, 32, 2)
#define DL_L(a, b, c, d) &launch_dl<a, b, c, d>
#define DL_O(a, b, c, d) &occ_dl<a, b, c, d>
#define DL_C(a, b, c, d) {a, b, c, d}
const DlLaunchFn kDlFns[] = {DL_CFGS(DL_L)};
const DlOccFn kDlOcc[] = {DL_CFGS(DL_O)};
constexpr int kDlCheck[][4] = {DL_CFGS(DL_C)};
constexpr bool dl_match() {
  for (int i = 0; i < N_DL_CFG; ++i)
    if (kDlCheck[i][0] != kDlCfg[i].bm || kDlCheck[i][1] != kDlCfg[i].bn || kDlCheck[i][2] != kDlCfg[i].bk ||
        kDlCheck[i][3] != kDlCfg[i].stages)
      return false;
  return true;
}
static_assert(sizeof(kDlFns) / sizeof(kDlFns[0]) == N_DL_CFG && dl_match(), "kernels must follow kDlCfg");
#define DL_W(a, b, c, d) Dl<a, b, c, d>::WPE
constexpr int kDlWpe[] = {DL_CFGS(DL_W)};
constexpr bool dl_occ_match() {
  for (int i = 0; i < N_DL_CFG; ++i)
    if (kDlWpe[i] != kDlCfg[i].occ) return false;
  return true;
}
static_assert(dl_occ_match(), "the table's workgroups per CU must be those the kernels are built for");

// the off-chip accumulation kernels: super-tiles of the 256 x 256 tiles
// (DL configurations 0 and 4), whose 512 KiB fp32 accumulator exceeds the
// registers
template <int BM, int BN, int BK, int S>
hipError_t launch_dl_sc(const Plan& p, const GemmArgs& g, hipStream_t st) {
  hipLaunchKernelGGL((k_dl_sc<BM, BN, BK, S>), dim3(p.grid_x, p.grid_y), dim3(256), 0, st, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dl_sc_main(const Plan& p, const GemmArgs& g, hipStream_t st) {
  const int cfg = p.cfg & 0xF, kc = 1 << (p.cfg >> 4);
  if (p.family != FAM_DLSC || (cfg != 0 && cfg != 4) || p.grid_y != kc || p.pk < 2 || p.pk % kc != 0 ||
      g.pk != p.pk || (int64_t)p.grid_x != (int64_t)((g.tiles_m + 1) / 2) * g.tiles_n || !ac::dl_operands_aligned(g))
    return hipErrorInvalidValue;
  return cfg == 0 ? launch_dl_sc<256, 256, 64, 2>(p, g, st) : launch_dl_sc<256, 256, 32, 4>(p, g, st);
}

hipError_t launch_dl_main(const Plan& p, const GemmArgs& g, hipStream_t st) {
  if (p.family != FAM_DL || p.cfg < 0 || p.cfg >= N_DL_CFG) return hipErrorInvalidValue;
  // the register-load form takes any alignment (K >= 8, N >= 8; two stages)
  if (p.unal ? (!kDlCfg[p.cfg].unal || g.K < 8 || g.N < 8) : !ac::dl_operands_aligned(g)) return hipErrorInvalidValue;
  if ((g.lay & ~kDlCfg[p.cfg].col) != 0) return hipErrorInvalidValue;
  return kDlFns[p.cfg](p, g, st, dtype_out16(p.s.dtype));
}

// The grouped kernel of a tile configuration in its direct-to-LDS form
// (where grouped_dl_runs; the register-staged one has the same bits).
hipError_t launch_grouped_dl_plan(const Plan& p, const GroupArgs& a, hipStream_t st) {
  if (!ac::grouped_dl_runs(p, a)) return hipErrorInvalidValue;
  const GemmArgs& g = a.g;
  GroupArgs b = a;
  b.g.kB = g.K;
  b.g.nB = g.N;
  const bool obf = dtype_out16(p.s.dtype);
  const TileCfg& t = kTileCfg[p.cfg];
  if (t.bm == 256 && t.bn == 128) return launch_grouped_dl<256, 128, 64, 3>(p, b, st, obf);
  if (t.bm == 128 && t.bn == 256) return launch_grouped_dl<128, 256, 64, 3>(p, b, st, obf);
  if (t.bm == 128 && t.bn == 128 && t.depth == 1) return launch_grouped_dl<128, 128, 64, 2>(p, b, st, obf);
  if (t.bm == 128 && t.bn == 128) return launch_grouped_dl<128, 128, 64, 3>(p, b, st, obf);
  if (t.bm == 64 && t.bn == 128) return launch_grouped_dl<64, 128, 64, 3>(p, b, st, obf);
  return hipErrorInvalidValue;
}

void query_occupancy_dl() {
  for (int i = 0; i < N_DL_CFG; ++i) set_runtime_occupancy(FAM_DL, i, kDlOcc[i]());
}

#endif  // AC_DL_PART

#if AC_INPUT_F16
}  // namespace f16
#elif AC_DL_PART == 0
bool dl_a_aligned(const void* A, int64_t lda, int64_t K) {
  return (reinterpret_cast<uintptr_t>(A) & 15) == 0 && (lda & 7) == 0 && (K & 7) == 0 && lda < DL_MAX_LD;
}
bool dl_b_aligned(const void* B, int64_t ldb, int64_t nB) {
  return (reinterpret_cast<uintptr_t>(B) & 15) == 0 && (ldb & 7) == 0 && (nB & 7) == 0 && ldb < DL_MAX_LD;
}
// Every group's operands must be aligned: the first one's, and the strides. A
// single k-block leaves nothing to pipeline: 96 products of 200 x 200 x 64 run
// in 6.5 us register-staged (128 x 64 tiles), 6.9 direct-to-LDS at best.
bool grouped_dl_aligned(const GroupArgs& a) {
  const GemmArgs& g = a.g;
  return g.K >= GROUPED_DL_MIN_K && dl_a_aligned(g.A, g.lda, g.K) && dl_b_aligned(g.B, g.ldb, g.N) &&
         (a.groups <= 1 || ((a.stride_a & 7) == 0 && (a.stride_b & 7) == 0));
}
bool grouped_dl_runs(const Plan& p, const GroupArgs& a) {
  return (p.family == FAM_GROUPED || p.family == FAM_BATCHED) && p.cfg >= 0 && p.cfg < N_TILE_CFG &&
         kGroupedDlStages[p.cfg] > 0 && grouped_dl_aligned(a);
}
// (an operand read in place column-major: rows of M, or of K)
bool dl_operands_aligned(const GemmArgs& g) {
  return ((g.lay & 1) ? dl_b_aligned(g.A, g.lda, g.M) : dl_a_aligned(g.A, g.lda, g.K)) &&
         ((g.lay & 2) ? dl_a_aligned(g.B, g.ldb, g.K) : dl_b_aligned(g.B, g.ldb, g.nB));
}

// ---- padding prologue (the Padding module of Table 2)
// dst (rows x ld_dst, ld_dst = cols rounded up to 8, 16-byte aligned) =
// src (rows x cols, row pitch ld_src, any 2-byte alignment), zeros in the pad
// columns: every row of the copy is a whole number of aligned 16-byte
// chunks. A thread moves one 16-byte group; x: groups of a row, y: rows.
__global__ __launch_bounds__(256) void k_pad16(const uint16_t* __restrict__ src, int64_t ld_src,
                                               uint16_t* __restrict__ dst, int64_t ld_dst, int64_t rows,
                                               int64_t cols) {
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= ld_dst) return;
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const uint16_t* s = src + r * ld_src + c;
    u32x4 v;
    if (c + 8 <= cols) {
      __builtin_memcpy(&v, s, 16);  // unaligned 16-byte load (gfx950 unaligned mode)
    } else {
      uint32_t h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = c + e < cols ? s[e] : 0u;
      v = u32x4{h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16)};
    }
    __builtin_memcpy(dst + r * ld_dst + c, &v, 16);
  }
}

hipError_t launch_pad16(const uint16_t* src, int64_t ld_src, int64_t rows, int64_t cols, uint16_t* dst,
                        int64_t ld_dst, hipStream_t st) {
  if (rows <= 0 || cols <= 0) return hipSuccess;
  if (ld_src < cols || ld_dst < cols || (ld_dst & 7) != 0 || ((uintptr_t)dst & 15) != 0) return hipErrorInvalidValue;
  const int64_t gx = (ld_dst / 8 + 255) / 256;
  if (gx > (1LL << 31) - 1) return hipErrorInvalidValue;
  const dim3 grid((unsigned)gx, (unsigned)(rows < 4096 ? rows : 4096)), block(256);
  hipLaunchKernelGGL(k_pad16, grid, block, 0, st, src, ld_src, dst, ld_dst, rows, cols);
  return hipGetLastError();
}
#endif
}  // namespace ac
