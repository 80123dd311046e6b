// gfx950 kernels of microscaled 4-bit matrices (mx_format.h): quantisation of
// rows, their values again, and products of few rows. (Products of more rows:
// kernels_mx_tile.hip.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ops.h"

namespace ac {
namespace {

#include "row_ops.h"
#include "mx_format.h"
#include "activations.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// s_waitcnt immediate for vmcnt(n) alone (expcnt 7 and lgkmcnt 15 do not wait; vmcnt
// bits 3:0 and 15:14)
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }

// i / d and i % d for i < 2^31 by a multiplication.
struct Division {
  uint32_t d, m, s;
  static Division by(uint32_t d) {  // 1 <= d < 2^31
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
  }
  __device__ __forceinline__ uint32_t quotient(uint32_t i) const { return (__umulhi(m, i) + i) >> s; }
};

// Elements c .. c+7 of a row of n, zeros past its end, with one load.
template <int T>
__device__ __forceinline__ void row8(const void* row, int64_t c, int64_t n, float (&f)[8]) {
  if (n < 8) {
    unpack<T>(load8<T>(row, (int)c, (int)n), f);
    return;
  }
  const int64_t at = min(c, n - 8);
  const int s = (int)min(c - at, (int64_t)8);
  Chunk<T> r;
  __builtin_memcpy(&r, static_cast<const char*>(row) + at * elem_bytes(T), sizeof r);
  unpack<T>(r, f);
  if (s != 0) {
#pragma unroll
    for (int step = 4; step >= 1; step >>= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (s & step) ? (e + step < 8 ? f[e + step] : 0.f) : f[e];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = s == 8 ? 0.f : f[e];
  }
}

// ---- quantisation of contiguous rows: a lane has eight values, a quad of
// lanes a block. Memory-bound: 2.5 bytes an element of 16 bits.
// QU: chunks a thread has in flight; one where the matrix is small, so that more
// CUs have a part of it (16 x 14336: 2.8 us, 4.5 with four). 1777 x 2731 of fp16 5.2
// us, 9.6 MB read and 2.6 written; 14336 x 4096 of bf16 26.0 (149 MB, 5.7 TB/s), of fp32
// 39.3 in a row and 46 from memory (266 MB); values again, 14336 x 4096 to bf16, 23.2 us
// (6.3 TB/s, of which the caches give the codes).
constexpr int QU = 4;
constexpr int64_t QU_SMALL = 1 << 18;  // chunks up to which one each
template <int T, int U>
__device__ __forceinline__ void quantise_chunks(const MxQuantArgs& a, const Division& per_row, int64_t row0, uint32_t n,
                                                uint32_t i0) {
  float f[U][8];
  int64_t row[U];
  uint32_t c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = i0 + u * 256, q = per_row.quotient(i);
    row[u] = row0 + q;
    c[u] = i - q * per_row.d;
    if (i < n) row8<T>(static_cast<const char*>(a.x) + row[u] * a.ldx * elem_bytes(T), (int64_t)c[u] * 8, a.cols, f[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (i0 + u * 256 >= n) break;  // (n is a multiple of four: whole quads)
    const uint32_t s = mx_scale_byte(mx_top_quad(mx_top8(f[u])));
    const uint32_t codes = mx_codes8(f[u], s), b = c[u] >> 2;
    int64_t at = row[u] * a.ld + (int64_t)c[u] * 4, scale_at = row[u] * a.lds + b;
    if (a.order == MX_IN_LANES) {
      const int64_t stage = (row[u] >> 4) * a.lds + (b >> 4);
      const int lane = (b & 12) * 4 + (int)(row[u] & 15);
      at = stage * 4096 + (b & 3) * 1024 + lane * 16 + (c[u] & 3) * 4;
      scale_at = stage * 256 + lane * 4 + (b & 3);
    } else if (a.order == MX_IN_STAGES) {
      scale_at = ((int64_t)(b >> 3) * a.lds + row[u]) * 8 + (b & 7);
    }
    __builtin_memcpy(a.codes + at, &codes, 4);
    if ((threadIdx.x & 3) == 0) a.scales[scale_at] = (uint8_t)s;
  }
}
template <int T, int U>
__global__ __launch_bounds__(256) void k_mx_quant(MxQuantArgs a, Division per_row, int64_t slab) {
  const int64_t row0 = (int64_t)blockIdx.y * slab;
  quantise_chunks<T, U>(a, per_row, row0, (uint32_t)min(slab, a.rows - row0) * per_row.d,
                        blockIdx.x * (256u * U) + threadIdx.x);
}

// ---- what products on tiles need done to their operands first, in one launch
// (4096 x 4096 and 14336 x 4096 in 4 bits: 2.4 MB of scales). A workgroup quantises
// 1024 chunks, or moves 32 rows of a matrix: their scales, to eight bytes of
// each stage, or their codes to aligned rows.
template <int T, int U>
__global__ __launch_bounds__(256) void k_mx_prepare(MxPrepare p, Division per_row, int quants) {
  const int b = blockIdx.x;
  if (b < quants) {
    quantise_chunks<T, U>(p.q, per_row, 0, (uint32_t)p.q.rows * per_row.d, (uint32_t)b * (256u * U) + threadIdx.x);
    return;
  }
  int k = 0, rest = b - quants;
  for (;; ++k) {
    const int n = (int)((p.m[k].rows + 31) / 32);
    if (rest < n) break;
    rest -= n;
  }
  const MxMove& m = p.m[k];
  const int64_t r0 = (int64_t)rest * 32;
  if (m.scales) {
    // eight lanes a row, 64 bytes of it
    const int64_t row = r0 + (threadIdx.x >> 3);
    const int stages = (m.bytes + 7) / 8;
    if (row < m.rows)
      for (int s = threadIdx.x & 7; s < stages; s += 8) {
        const uint8_t* src = m.src + row * m.ld + s * 8;
        uint64_t v = 0;
        if (s * 8 + 8 <= m.bytes) {
          __builtin_memcpy(&v, src, 8);
        } else {
          for (int e = 0; e < 7; ++e)
            if (s * 8 + e < m.bytes) v |= (uint64_t)src[e] << (8 * e);
        }
        *reinterpret_cast<uint64_t*>(m.dst + ((int64_t)s * m.ldd + row) * 8) = v;
      }
    return;
  }
  const int64_t row = r0 + (threadIdx.x >> 3);
  if (row < m.rows)
    for (int c = (threadIdx.x & 7) * 16; c < m.bytes; c += 128) {  // (codes: whole blocks)
      u32x4 v;
      __builtin_memcpy(&v, m.src + row * m.ld + c, 16);
      *reinterpret_cast<u32x4*>(m.dst + row * m.ldd + c) = v;
    }
}

// ---- quantisation of a transposed view: element (r, c) at c ldx + r, blocks
// along c. A lane takes two neighbouring r and the 32 c of a block, a wave 128 r
// of two blocks, a workgroup a tile of 128 r x 8 blocks, which goes through LDS
// so that a row's 128 bytes of codes leave together. Memory-bound: 14336 x 4096 of
// bf16 28.0 us (149 MB, 5.3 TB/s). Not so fp32: its copy of a length known only when it
// runs keeps the 64 values in scratch memory (272 bytes a lane): 433 us for the 266 MB
// that take 39 as rows.
template <int T>
__global__ __launch_bounds__(256) void k_mx_quant_t(MxQuantArgs a) {
  constexpr int LD = 8 * MX_BYTES + 16;
  __shared__ __attribute__((aligned(16))) uint8_t codes[128 * LD];
  __shared__ __attribute__((aligned(16))) uint8_t scales[128 * 8];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)blockIdx.x * 128, blk0 = (int64_t)blockIdx.y * 8, blocks = (a.cols + 31) / 32;
  // the lane's pair of rows: the last two where it would pass the end
  const int64_t r = min(r0 + 2 * lane, a.rows > 1 ? a.rows - 2 : 0);
  const int at = (int)(r - r0);  // (-1: the tile has one row left)
#pragma unroll 1
  for (int b = 2 * w; b < 2 * w + 2; ++b) {
    const int64_t c0 = (blk0 + b) * 32;
    if (blk0 + b >= blocks) break;
    uint32_t raw[T == AC_TYPE_F32 ? 64 : 32];
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const char* p = static_cast<const char*>(a.x) + ((c0 + k) * a.ldx + r) * elem_bytes(T);
      if constexpr (T == AC_TYPE_F32) {
        raw[2 * k] = raw[2 * k + 1] = 0;
        if (c0 + k < a.cols) __builtin_memcpy(&raw[2 * k], p, a.rows > 1 ? 8 : 4);
      } else {
        raw[k] = 0;
        if (c0 + k < a.cols) {
          if (a.rows > 1)
            __builtin_memcpy(&raw[k], p, 4);
          else
            raw[k] = *reinterpret_cast<const uint16_t*>(p);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t top = 0, out[4];
      auto value = [&](int k) {
        if constexpr (T == AC_TYPE_F32) return __uint_as_float(raw[2 * k + h]);
        const uint32_t v = h ? raw[k] >> 16 : raw[k] & 0xFFFFu;
        if constexpr (T == AC_TYPE_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)v);
        return __uint_as_float(v << 16);
      };
#pragma unroll
      for (int k = 0; k < 32; ++k) top = max(top, __float_as_uint(value(k)) & 0x7FFFFFFFu);
      const uint32_t s = mx_scale_byte(top);
#pragma unroll
      for (int o = 0; o < 4; ++o) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = value(8 * o + e);
        out[o] = mx_codes8(f, s);
      }
      if (at + h >= 0) {
        *reinterpret_cast<u32x4*>(codes + (at + h) * LD + b * MX_BYTES) = u32x4{out[0], out[1], out[2], out[3]};
        scales[(at + h) * 8 + b] = (uint8_t)s;
      }
    }
  }
  __syncthreads();
  const int b = threadIdx.x & 7;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = (threadIdx.x >> 3) + 32 * i;
    if (r0 + t < a.rows && blk0 + b < blocks) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(codes + t * LD + b * MX_BYTES);
      __builtin_memcpy(a.codes + (r0 + t) * a.ld + (blk0 + b) * MX_BYTES, &v, 16);
      a.scales[(r0 + t) * a.lds + blk0 + b] = scales[t * 8 + b];
    }
  }
}

// ---- the values again
template <int T, int U>
__global__ __launch_bounds__(256) void k_mx_dequant(MxDequantArgs a, Division per_row, int64_t slab) {
  const int64_t row0 = (int64_t)blockIdx.y * slab;
  const uint32_t n = (uint32_t)min(slab, a.rows - row0) * per_row.d;
  const uint32_t i0 = blockIdx.x * (256u * U) + threadIdx.x;
  uint32_t codes[U], s[U], c[U];
  int64_t row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = i0 + u * 256, q = per_row.quotient(i);
    row[u] = row0 + q;
    c[u] = i - q * per_row.d;
    if (i < n) {
      __builtin_memcpy(&codes[u], a.m.codes + row[u] * a.m.ld + (int64_t)c[u] * 4, 4);
      s[u] = a.m.scales[row[u] * a.m.lds + (c[u] >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (i0 + u * 256 >= n) break;
    float f[8];
    mx_values8(codes[u], s[u], f);
    store8<T>(static_cast<char*>(a.y) + row[u] * a.ldy * elem_bytes(T), (int)(c[u] * 8), (int)a.cols, f);
  }
}

// ---- few rows: a workgroup takes 16 rows of B and MT * 16 of A; its SW waves take
// stages of 512 k in turn. A lane of the matrix instruction has 16 bytes, a block, of
// row lane % 16, so that neighbouring lanes are in different rows: loaded straight
// into registers that costs an address a lane (16 x 4096 x 14336: 15.8 us, 2.0 TB/s).
// Instead a stage's 256 bytes of a row are loaded by 16 neighbouring lanes into LDS
// of the wave's own (no barriers, two stages in flight), the 16-byte chunks swizzled
// with the row. Lane quarter q takes blocks 4 q .. 4 q + 3 of a stage in its four
// instructions, so that its scales are four bytes next to each other; B is read
// once, A, small, by every workgroup from the caches. TX >= 0: A is not quantised
// yet; every workgroup does it, into LDS, while its first loads of B are on their
// way: a launch less. TX == LANES: a launch before this one has quantised A and left
// it in the lanes' order: it goes straight to registers, and its place in LDS to a
// second workgroup of the CU. Memory-bound where B is large: 16 x 14336 x 4096 gated
// 12.7 us (62 MB, 4.9 TB/s; 17.3 with A's codes through LDS), 16 x 4096 x 14336 6.1 us
// (31 MB, 5.1 TB/s; 6.8); one row of 4096 x 4096 4.1 us, half of it the start of the
// launch and the loads' first round trip.
constexpr int CODES = -1, LANES = -2;
typedef __attribute__((address_space(3))) void lds_void;
constexpr int32_t OOB_OFF = (int32_t)0x80000000u;  // past every range: reads zeros
__device__ __forceinline__ void load_lds16(const uint8_t* base, int32_t off, uint8_t* lds) {
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), (short)0, (int)0x7FFFFFF0, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)lds, 16, off, 0, 0, 0);
}
template <int KS>
__device__ __forceinline__ f32x4 mx_mfma16(u32x4 a, uint32_t sa, u32x4 b, uint32_t sb, f32x4 c) {
  const i32x8 va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, KS, (int)sa, KS, (int)sb);
}
// Scale bytes blk .. blk + 3 of a row of n (zeros past its end), at any address.
__device__ __forceinline__ uint32_t scales4(const uint8_t* row, int blk, int n) {
  uint32_t v = 0;
  if (blk + 4 <= n) {
    __builtin_memcpy(&v, row + blk, 4);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (blk + e < n) v |= (uint32_t)row[blk + e] << (8 * e);
  }
  return v;
}

// LDS of a quantised A: rows of codes 16 bytes apart from whole banks, then the
// scales of all rows.
__host__ __device__ constexpr int64_t rows_lds_pitch(int64_t blocks) { return blocks * MX_BYTES + 16; }
__host__ __device__ constexpr int64_t rows_lds_bytes(int64_t M, int64_t blocks) {
  return M * rows_lds_pitch(blocks) + M * blocks;
}

// Sums of the waves in `part` (the workgroup's outputs MT * 256 a product and wave),
// in their order, and what leaves.
template <int MT, int SW, bool GATED>
__device__ __forceinline__ void rows_out(const MxProduct& g, const float* part, int64_t m0, int64_t n0) {
  constexpr int NB = GATED ? 2 : 1;
  for (int i = threadIdx.x; i < MT * 256; i += 64 * SW) {
    const int64_t row = m0 + (i >> 4), c = n0 + (i & 15);
    if (row >= g.M || c >= g.N) continue;
    float v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      v[j] = part[j * MT * 256 + i];
#pragma unroll
      for (int k = 1; k < SW; ++k) v[j] += part[(k * NB + j) * MT * 256 + i];
    }
    float o = GATED ? act1(g.act, v[0]) * v[NB - 1] : v[0];
    if (!GATED && g.bias) o += g.bias[c];
    if (g.out_type == AC_TYPE_F32)
      put<AC_TYPE_F32>(g.out, row * g.ldo + c, o);
    else if (g.out_type == AC_TYPE_F16)
      put<AC_TYPE_F16>(g.out, row * g.ldo + c, o);
    else
      put<AC_TYPE_BF16>(g.out, row * g.ldo + c, o);
  }
}
// A quantised into LDS by the workgroup, four chunks a thread at a time.
template <int SW, int TX>
__device__ __forceinline__ void rows_quantise(const MxProduct& g, const MxQuantArgs& x, const Division& per_row,
                                              uint8_t* qa) {
  const int pitch = (int)rows_lds_pitch(g.blocks);
  const uint32_t n = (uint32_t)g.M * per_row.d;  // (a multiple of four: a quad of lanes a block)
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += 64 * SW * QU) {
    float f[QU][8];
    int r[QU], c[QU];
#pragma unroll
    for (int u = 0; u < QU; ++u) {
      const uint32_t i = i0 + u * 64 * SW;
      r[u] = (int)per_row.quotient(i);
      c[u] = (int)(i - r[u] * per_row.d);
      if (i < n) row8<TX>(static_cast<const char*>(x.x) + r[u] * x.ldx * elem_bytes(TX), (int64_t)c[u] * 8, x.cols, f[u]);
    }
#pragma unroll
    for (int u = 0; u < QU; ++u) {
      if (i0 + u * 64 * SW >= n) break;
      const uint32_t sc = mx_scale_byte(mx_top_quad(mx_top8(f[u])));
      *reinterpret_cast<uint32_t*>(qa + r[u] * pitch + c[u] * 4) = mx_codes8(f[u], sc);
      if ((c[u] & 3) == 0) qa[(int)g.M * pitch + r[u] * g.blocks + (c[u] >> 2)] = (uint8_t)sc;
    }
  }
}

// DIRECT: B (and A) can be loaded into LDS (16-byte aligned codes and pitches);
// otherwise straight into registers, any alignment (gated, with 32 rows of codes,
// 68 bytes a lane lie in scratch memory).
template <int MT, int SW, bool GATED, int TX, bool DIRECT>
__global__ __launch_bounds__(64 * SW) void k_mx_rows(MxProduct g, MxQuantArgs x, Division per_row) {
  constexpr int NB = GATED ? 2 : 1;
  constexpr bool LDSA = TX >= 0, INREGS = TX == LANES || !DIRECT;
  constexpr int TILES = (TX == CODES ? MT : 0) + NB, STAGE = TILES * 4096;  // a stage of a wave: 16 rows of 256 bytes each
  __shared__ __attribute__((aligned(16))) uint8_t st0[DIRECT ? SW * STAGE : 16];
  __shared__ __attribute__((aligned(16))) uint8_t st1[DIRECT ? SW * STAGE : 16];
  __shared__ __attribute__((aligned(16))) float part[SW * NB * MT * 256];
  extern __shared__ __attribute__((aligned(16))) uint8_t qa[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, quarter = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (MT * 16);
  const int nst = (g.blocks + 15) / 16;
  // the lane's rows (past the end: the last one again, what it gives goes nowhere)
  const int64_t nr = min(n0 + i16, g.N - 1);
  const uint8_t *bs[NB], *as[MT], *bc[NB], *ac_[MT];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    bs[j] = (j ? g.b2.scales : g.b.scales) + nr * g.b.lds;
    bc[j] = (j ? g.b2.codes : g.b.codes) + nr * g.b.ld;
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t mr = min(m0 + m * 16 + i16, g.M - 1);
    as[m] = LDSA ? qa + g.M * rows_lds_pitch(g.blocks) + mr * g.blocks : g.a.scales + mr * g.a.lds;
    ac_[m] = LDSA ? qa + mr * rows_lds_pitch(g.blocks) : g.a.codes + mr * g.a.ld;
  }
  // the lane's chunks of a stage's loads into LDS: row 4 q + lane / 16 of a tile,
  // slot lane % 16 (holding chunk slot ^ row)
  int32_t off_b[4], off_a[4 * MT];
  int chunk[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = 4 * q + (lane >> 4);
    chunk[q] = (lane & 15) ^ r;
    off_b[q] = n0 + r < g.N ? (int32_t)(r * g.b.ld) + chunk[q] * MX_BYTES : OOB_OFF;
#pragma unroll
    for (int m = 0; m < MT; ++m)
      off_a[4 * m + q] = m0 + m * 16 + r < g.M ? (int32_t)((m * 16 + r) * g.a.ld) + chunk[q] * MX_BYTES : OOB_OFF;
  }
  f32x4 acc[NB][MT];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[j][m] = f32x4{};
  struct Regs {
    uint32_t sb[NB], sa[MT];
    u32x4 b[DIRECT ? 1 : 4][NB], a[INREGS ? 4 : 1][MT];
  };
  const auto issue = [&](Regs& v, uint8_t* st, int s) {
    uint8_t* const to = st + w * STAGE;
    const int blk = s * 16 + 4 * quarter;
    if constexpr (DIRECT) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bool in = s * 16 + chunk[q] < g.blocks;
#pragma unroll
        for (int j = 0; j < NB; ++j)
          load_lds16((j ? g.b2.codes : g.b.codes) + n0 * g.b.ld + (int64_t)s * 256, in ? off_b[q] : OOB_OFF,
                     to + j * 4096 + q * 1024);
        if constexpr (TX == CODES) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
            load_lds16(g.a.codes + m0 * g.a.ld + (int64_t)s * 256, in ? off_a[4 * m + q] : OOB_OFF,
                       to + (NB + m) * 4096 + q * 1024);
        }
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          v.b[DIRECT ? 0 : ks][j] = u32x4{};
          if (blk + ks < g.blocks) __builtin_memcpy(&v.b[DIRECT ? 0 : ks][j], bc[j] + (int64_t)(blk + ks) * MX_BYTES, 16);
        }
        if constexpr (TX == CODES) {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            v.a[INREGS ? ks : 0][m] = u32x4{};
            if (blk + ks < g.blocks) __builtin_memcpy(&v.a[INREGS ? ks : 0][m], ac_[m] + (int64_t)(blk + ks) * MX_BYTES, 16);
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) v.sb[j] = scales4(bs[j], blk, g.blocks);
    if constexpr (TX == LANES) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int64_t stage = ((int64_t)blockIdx.y * MT + m) * nst + s;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          v.a[INREGS ? ks : 0][m] = *reinterpret_cast<const u32x4*>(g.a.codes + stage * 4096 + ks * 1024 + lane * 16);
        v.sa[m] = *reinterpret_cast<const uint32_t*>(g.a.scales + stage * 256 + lane * 4);
      }
    }
    if constexpr (TX == CODES) {
#pragma unroll
      for (int m = 0; m < MT; ++m) v.sa[m] = scales4(as[m], blk, g.blocks);
    }
  };
  const auto multiply = [&](Regs& v, const uint8_t* st, int s) {
    const uint8_t* const from = st + w * STAGE + i16 * 256;
    const int blk = s * 16 + 4 * quarter;
    if constexpr (LDSA) {
#pragma unroll
      for (int m = 0; m < MT; ++m) v.sa[m] = scales4(as[m], blk, g.blocks);
    }
    const auto one = [&](auto kc) {
      constexpr int ks = decltype(kc)::value;
      const int at = ((4 * quarter + ks) ^ i16) * MX_BYTES;
      u32x4 b[NB], a[MT];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if constexpr (DIRECT)
          b[j] = *reinterpret_cast<const u32x4*>(from + j * 4096 + at);
        else
          b[j] = v.b[DIRECT ? 0 : ks][j];
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if constexpr (LDSA) {
          a[m] = u32x4{};
          if (blk + ks < g.blocks) a[m] = *reinterpret_cast<const u32x4*>(ac_[m] + (blk + ks) * MX_BYTES);
        } else if constexpr (INREGS) {
          a[m] = v.a[INREGS ? ks : 0][m];
        } else {
          a[m] = *reinterpret_cast<const u32x4*>(from + (NB + m) * 4096 + at);
        }
      }
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[j][m] = mx_mfma16<ks>(b[j], v.sb[j], a[m], v.sa[m], acc[j][m]);
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
    one(std::integral_constant<int, 3>{});
  };
  // waits until at most N of the wave's loads are in flight (they end in their order)
  constexpr int LOADS = DIRECT ? 4 * TILES + NB + (TX == LANES ? 5 * MT : LDSA ? 0 : MT) : 0;
  const auto landed = [&](auto more) {
    if constexpr (DIRECT) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(decltype(more)::value ? LOADS : 0));
      asm volatile("" ::: "memory");
    }
  };
  // waits until the wave has what it read of a stage: new loads into it may land
  // before reads that were sent first (zeros, past a row's end, in no time)
  const auto have_read = [&] {
    if constexpr (DIRECT) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  // the wave's stages w, w + SW, ..., a pair at a time while there are more than two.
  // (As an endless loop left in the middle the compiler has been seen to carry one of
  // the four elements of a sum into it and to lose the others.)
  int s = w;
  Regs p, q;
  if (s < nst) issue(p, st0, s);
  if constexpr (LDSA) {
    rows_quantise<SW, TX>(g, x, per_row, qa);
    __syncthreads();
  }
  for (; s + 2 * SW < nst; s += 2 * SW) {
    issue(q, st1, s + SW);
    landed(std::true_type{});
    multiply(p, st0, s);
    have_read();
    issue(p, st0, s + 2 * SW);
    landed(std::true_type{});
    multiply(q, st1, s + SW);
    have_read();
  }
  if (s + SW < nst) {
    issue(q, st1, s + SW);
    landed(std::true_type{});
    multiply(p, st0, s);
    landed(std::false_type{});
    multiply(q, st1, s + SW);
  } else if (s < nst) {
    landed(std::false_type{});
    multiply(p, st0, s);
  }
  // a lane has row i16 and four columns of it
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m)
      *reinterpret_cast<f32x4*>(part + ((w * NB + j) * MT + m) * 256 + i16 * 16 + quarter * 4) = acc[j][m];
  __syncthreads();
  rows_out<MT, SW, GATED>(g, part, m0, n0);
}
template <int MT, bool GATED, int TX>
void start_rows(const MxProduct& p, const MxQuantArgs& x, int waves, bool direct, dim3 grid, hipStream_t st) {
  const size_t lds = TX >= 0 ? (size_t)rows_lds_bytes(p.M, p.blocks) : 0;
  const Division per = Division::by((uint32_t)(p.blocks > 0 ? p.blocks * 4 : 1));
  constexpr int TILES = (TX == CODES ? MT : 0) + (GATED ? 2 : 1), MOST = TILES * 8 * 8192 > 128 * 1024 || (TX >= 0 && TILES > 1) ? 4 : 8;
  if (!direct)
    hipLaunchKernelGGL((k_mx_rows<MT, 8, GATED, TX, false>), grid, dim3(512), lds, st, p, x, per);
  else if (waves >= MOST)
    hipLaunchKernelGGL((k_mx_rows<MT, MOST, GATED, TX, true>), grid, dim3(64 * MOST), lds, st, p, x, per);
  else
    hipLaunchKernelGGL((k_mx_rows<MT, 4, GATED, TX, true>), grid, dim3(256), lds, st, p, x, per);
}

// Rows a launch's chunk numbers reach, its grid and its division.
struct Chunks {
  Division per_row;
  int64_t slab;
  dim3 grid;
  int u;
  bool ok;
  Chunks(int64_t rows, int64_t cols, MxOrder order = MX_IN_ROWS) {
    // (whole stages: the scales of the blocks that are not there are zeros)
    const int64_t part = order == MX_IN_ROWS ? 32 : order == MX_IN_STAGES ? 256 : 512;
    const int64_t per = (cols + part - 1) / part * (part / 8);
    ok = per < (1LL << 30);
    if (!ok) return;
    slab = std::min<int64_t>(rows, ((1LL << 31) - 4096) / per);
    u = rows * per <= QU_SMALL ? 1 : QU;
    const int64_t x = (slab * per + 256 * u - 1) / (256 * u), y = (rows + slab - 1) / slab;
    ok = y <= 65535;
    per_row = Division::by((uint32_t)per);
    grid = dim3((unsigned)x, (unsigned)y);
  }
};

}  // namespace

#define MX_LAUNCH(k, T, grid, ...)                                                   \
  if (u == 1)                                                                      \
    hipLaunchKernelGGL((k<T, 1>), grid, dim3(256), 0, st, __VA_ARGS__);            \
  else                                                                             \
    hipLaunchKernelGGL((k<T, QU>), grid, dim3(256), 0, st, __VA_ARGS__)
#define MX_TYPES(k, grid, ...)                   \
  if (type == AC_TYPE_F32) {                     \
    MX_LAUNCH(k, AC_TYPE_F32, grid, __VA_ARGS__);  \
  } else if (type == AC_TYPE_F16) {              \
    MX_LAUNCH(k, AC_TYPE_F16, grid, __VA_ARGS__);  \
  } else {                                       \
    MX_LAUNCH(k, AC_TYPE_BF16, grid, __VA_ARGS__); \
  }
hipError_t launch_mx_quantize(const MxQuantArgs& a, int type, bool cols_contiguous, hipStream_t st) {
  if (a.rows < 1 || a.cols < 1) return hipSuccess;
  if (cols_contiguous) {
    const int64_t x = (a.rows + 127) / 128, y = (a.cols + 255) / 256;
    if (x >= (1LL << 31) / 256 || y > 65535) return hipErrorInvalidValue;
    const dim3 grid((unsigned)x, (unsigned)y);
    if (type == AC_TYPE_F32)
      hipLaunchKernelGGL((k_mx_quant_t<AC_TYPE_F32>), grid, dim3(256), 0, st, a);
    else if (type == AC_TYPE_BF16)
      hipLaunchKernelGGL((k_mx_quant_t<AC_TYPE_BF16>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((k_mx_quant_t<AC_TYPE_F16>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
  }
  const Chunks c(a.rows, a.cols, a.order);
  if (!c.ok) return hipErrorInvalidValue;
  const int u = c.u;
  MX_TYPES(k_mx_quant, c.grid, a, c.per_row, c.slab)
  return hipGetLastError();
}
hipError_t launch_mx_prepare(MxPrepare p, int type, hipStream_t st, int* launches) {
  int64_t blocks = 0;
  int u = QU;
  Division per = Division::by(4);
  if (p.q.x) {
    const Chunks c(p.q.rows, p.q.cols, p.q.order);
    if (!c.ok) return hipErrorInvalidValue;
    if (c.grid.y > 1) {  // more chunks than one division counts
      ++*launches;
      const hipError_t e = launch_mx_quantize(p.q, type, false, st);
      if (e != hipSuccess) return e;
      p.q.x = nullptr;
    } else {
      per = c.per_row;
      blocks = c.grid.x;
      u = c.u;
    }
  }
  const int64_t quants = blocks;
  for (int i = 0; i < p.n; ++i) blocks += (p.m[i].rows + 31) / 32;
  if (blocks >= (1LL << 31) / 256) return hipErrorInvalidValue;
  if (blocks == 0) return hipSuccess;
  ++*launches;
  const dim3 grid((unsigned)blocks);
  if (!p.q.x) type = AC_TYPE_BF16;  // (any: nothing is quantised)
  MX_TYPES(k_mx_prepare, grid, p, per, (int)quants)
  return hipGetLastError();
}
hipError_t launch_mx_dequantize(const MxDequantArgs& a, int type, hipStream_t st) {
  if (a.rows < 1 || a.cols < 1) return hipSuccess;
  const Chunks c(a.rows, a.cols);
  if (!c.ok) return hipErrorInvalidValue;
  const int u = c.u;
  MX_TYPES(k_mx_dequant, c.grid, a, c.per_row, c.slab)
  return hipGetLastError();
}
int64_t mx_rows_lds(int64_t M, int64_t blocks) { return rows_lds_bytes(M, blocks); }
hipError_t launch_mx_rows(const MxProduct& p, bool gated, const MxQuantArgs* x, int type, bool lanes, int waves,
                          bool direct, hipStream_t st) {
  if (p.M < 1 || p.N < 1) return hipErrorInvalidValue;
  const bool two = p.M > 16;
  const int64_t y = two ? (p.M + 31) / 32 : 1, gx = (p.N + 15) / 16;
  if (y > 65535 || gx >= (1LL << 31) / 512 || (x && (two || rows_lds_bytes(p.M, p.blocks) > MX_ROWS_LDS)))
    return hipErrorInvalidValue;
  const dim3 grid((unsigned)gx, (unsigned)y);
  const MxQuantArgs q = x ? *x : MxQuantArgs{};
#define MX_ROWS(MT, T) \
  gated ? start_rows<MT, true, T>(p, q, waves, direct, grid, st) : start_rows<MT, false, T>(p, q, waves, direct, grid, st)
  if (two && lanes)
    MX_ROWS(2, LANES);
  else if (two)
    MX_ROWS(2, CODES);
  else if (lanes)
    MX_ROWS(1, LANES);
  else if (!x)
    MX_ROWS(1, CODES);
  else if (type == AC_TYPE_BF16)
    MX_ROWS(1, AC_TYPE_BF16);
  else if (type == AC_TYPE_F16)
    MX_ROWS(1, AC_TYPE_F16);
  else
    MX_ROWS(1, AC_TYPE_F32);
#undef MX_ROWS
  return hipGetLastError();
}

}  // namespace ac
