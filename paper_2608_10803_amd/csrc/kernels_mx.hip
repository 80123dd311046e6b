// gfx950 kernels of microscaled 4-bit matrices (mx_format.h): quantisation of
// rows, their values again, and products of few rows. (Products of more rows:
// kernels_mx_tile.hip.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ops.h"

namespace ac {
namespace {

#include "row_ops.h"
#include "mx_format.h"
#include "activations.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

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
constexpr int QU = 4;  // chunks a thread has in flight
template <int T>
__global__ __launch_bounds__(256) void k_mx_quant(MxQuantArgs a, Division per_row, int64_t slab) {
  const int64_t row0 = (int64_t)blockIdx.y * slab;
  const uint32_t n = (uint32_t)min(slab, a.rows - row0) * per_row.d;
  const uint32_t i0 = blockIdx.x * (256u * QU) + threadIdx.x;
  float f[QU][8];
  int64_t row[QU];
  uint32_t c[QU];
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint32_t i = i0 + u * 256, q = per_row.quotient(i);
    row[u] = row0 + q;
    c[u] = i - q * per_row.d;
    if (i < n) row8<T>(static_cast<const char*>(a.x) + row[u] * a.ldx * elem_bytes(T), (int64_t)c[u] * 8, a.cols, f[u]);
  }
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    if (i0 + u * 256 >= n) break;  // (n is a multiple of four: whole quads)
    const uint32_t s = mx_scale_byte(mx_top_quad(mx_top8(f[u])));
    const uint32_t codes = mx_codes8(f[u], s);
    __builtin_memcpy(a.codes + row[u] * a.ld + (int64_t)c[u] * 4, &codes, 4);
    if ((threadIdx.x & 3) == 0) a.scales[row[u] * a.lds + (c[u] >> 2)] = (uint8_t)s;
  }
}

// ---- quantisation of a transposed view: element (r, c) at c ldx + r, blocks
// along c. A lane takes two neighbouring r and the 32 c of a block, a wave 128 r
// of two blocks, a workgroup a tile of 128 r x 8 blocks, which goes through LDS
// so that a row's 128 bytes of codes leave together.
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
template <int T>
__global__ __launch_bounds__(256) void k_mx_dequant(MxDequantArgs a, Division per_row, int64_t slab) {
  const int64_t row0 = (int64_t)blockIdx.y * slab;
  const uint32_t n = (uint32_t)min(slab, a.rows - row0) * per_row.d;
  const uint32_t i0 = blockIdx.x * (256u * QU) + threadIdx.x;
  uint32_t codes[QU], s[QU], c[QU];
  int64_t row[QU];
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    const uint32_t i = i0 + u * 256, q = per_row.quotient(i);
    row[u] = row0 + q;
    c[u] = i - q * per_row.d;
    if (i < n) {
      __builtin_memcpy(&codes[u], a.m.codes + row[u] * a.m.ld + (int64_t)c[u] * 4, 4);
      s[u] = a.m.scales[row[u] * a.m.lds + (c[u] >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < QU; ++u) {
    if (i0 + u * 256 >= n) break;
    float f[8];
    mx_values8(codes[u], s[u], f);
    store8<T>(static_cast<char*>(a.y) + row[u] * a.ldy * elem_bytes(T), (int)(c[u] * 8), (int)a.cols, f);
  }
}

// ---- few rows: a workgroup takes 16 rows of B and MT * 16 of A; its SW waves
// take 128 k each in turn, straight from memory into the operands of one matrix
// instruction: a lane has 16 bytes, a block of a row, and its scale byte. Any
// alignment, any number of blocks.
__device__ __forceinline__ f32x4 mx_mfma16(u32x4 a, uint32_t sa, u32x4 b, uint32_t sb, f32x4 c) {
  const i32x8 va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, 0, (int)sa, 0, (int)sb);
}

template <int MT, int SW, bool GATED>
__global__ __launch_bounds__(64 * SW) void k_mx_rows(MxProduct g) {
  constexpr int NB = GATED ? 2 : 1, U = 2;
  __shared__ __attribute__((aligned(16))) float part[SW * NB * MT * 256];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, quarter = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (MT * 16);
  const uint8_t *b[NB], *bs[NB], *x[MT], *xs[MT];
  const int64_t nr = min(n0 + i16, g.N - 1);
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    b[j] = (j ? g.b2.codes : g.b.codes) + nr * g.b.ld;
    bs[j] = (j ? g.b2.scales : g.b.scales) + nr * g.b.lds;
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {  // (rows past the end repeat the last; what they give goes nowhere)
    const int64_t mr = min(m0 + m * 16 + i16, g.M - 1);
    x[m] = g.a.codes + mr * g.a.ld;
    xs[m] = g.a.scales + mr * g.a.lds;
  }
  f32x4 acc[NB][MT];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[j][m] = f32x4{};
  struct Batch {
    u32x4 b[U][NB], x[U][MT];
    uint32_t bs[U][NB], xs[U][MT];
  };
  auto load = [&](Batch& v, int s) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int blk = (s + u * SW) * 4 + quarter;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        v.b[u][j] = u32x4{};
        v.bs[u][j] = 0;
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        v.x[u][m] = u32x4{};
        v.xs[u][m] = 0;
      }
      if (blk >= g.blocks) continue;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        __builtin_memcpy(&v.b[u][j], b[j] + (int64_t)blk * MX_BYTES, 16);
        v.bs[u][j] = bs[j][blk];
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        __builtin_memcpy(&v.x[u][m], x[m] + (int64_t)blk * MX_BYTES, 16);
        v.xs[u][m] = xs[m][blk];
      }
    }
  };
  auto multiply = [&](const Batch& v) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int m = 0; m < MT; ++m)
          acc[j][m] = mx_mfma16(v.b[u][j], v.bs[u][j], v.x[u][m], v.xs[u][m], acc[j][m]);
  };
  const int steps = (g.blocks + 3) / 4;
  Batch p;
  for (int s = w; s < steps; s += U * SW) {
    load(p, s);
    multiply(p);
  }
  // a lane has row i16 and four columns of it; the waves' sums are added in
  // their order
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m)
      *reinterpret_cast<f32x4*>(part + ((w * NB + j) * MT + m) * 256 + i16 * 16 + quarter * 4) = acc[j][m];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += 64 * SW) {
    const int64_t row = m0 + (i >> 4), c = n0 + (i & 15);
    if (row >= g.M || c >= g.N) continue;
    float v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      v[j] = part[j * MT * 256 + i];
#pragma unroll
      for (int q = 1; q < SW; ++q) v[j] += part[(q * NB + j) * MT * 256 + i];
    }
    float o = GATED ? act1(g.act, v[0]) * v[NB - 1] : v[0];
    if (g.bias) o += g.bias[c];
    if (g.out_type == AC_TYPE_F32)
      put<AC_TYPE_F32>(g.out, row * g.ldo + c, o);
    else if (g.out_type == AC_TYPE_F16)
      put<AC_TYPE_F16>(g.out, row * g.ldo + c, o);
    else
      put<AC_TYPE_BF16>(g.out, row * g.ldo + c, o);
  }
}

// Rows a launch's chunk numbers reach, its grid and its division.
struct Chunks {
  Division per_row;
  int64_t slab;
  dim3 grid;
  bool ok;
  Chunks(int64_t rows, int64_t cols) {
    const int64_t per = (cols + 31) / 32 * 4;
    ok = per < (1LL << 30);
    if (!ok) return;
    slab = std::min<int64_t>(rows, ((1LL << 31) - 4096) / per);
    const int64_t x = (slab * per + 256 * QU - 1) / (256 * QU), y = (rows + slab - 1) / slab;
    ok = y <= 65535;
    per_row = Division::by((uint32_t)per);
    grid = dim3((unsigned)x, (unsigned)y);
  }
};

}  // namespace

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
  const Chunks c(a.rows, a.cols);
  if (!c.ok) return hipErrorInvalidValue;
  if (type == AC_TYPE_F32)
    hipLaunchKernelGGL((k_mx_quant<AC_TYPE_F32>), c.grid, dim3(256), 0, st, a, c.per_row, c.slab);
  else if (type == AC_TYPE_BF16)
    hipLaunchKernelGGL((k_mx_quant<AC_TYPE_BF16>), c.grid, dim3(256), 0, st, a, c.per_row, c.slab);
  else
    hipLaunchKernelGGL((k_mx_quant<AC_TYPE_F16>), c.grid, dim3(256), 0, st, a, c.per_row, c.slab);
  return hipGetLastError();
}
hipError_t launch_mx_dequantize(const MxDequantArgs& a, int type, hipStream_t st) {
  if (a.rows < 1 || a.cols < 1) return hipSuccess;
  const Chunks c(a.rows, a.cols);
  if (!c.ok) return hipErrorInvalidValue;
  if (type == AC_TYPE_F32)
    hipLaunchKernelGGL((k_mx_dequant<AC_TYPE_F32>), c.grid, dim3(256), 0, st, a, c.per_row, c.slab);
  else if (type == AC_TYPE_BF16)
    hipLaunchKernelGGL((k_mx_dequant<AC_TYPE_BF16>), c.grid, dim3(256), 0, st, a, c.per_row, c.slab);
  else
    hipLaunchKernelGGL((k_mx_dequant<AC_TYPE_F16>), c.grid, dim3(256), 0, st, a, c.per_row, c.slab);
  return hipGetLastError();
}
hipError_t launch_mx_rows(const MxProduct& p, bool gated, hipStream_t st) {
  if (p.M < 1 || p.N < 1) return hipErrorInvalidValue;
  const int64_t y = (p.M + 31) / 32;
  if (y > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((p.N + 15) / 16), (unsigned)y);
  if (gated)
    hipLaunchKernelGGL((k_mx_rows<2, 4, true>), grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((k_mx_rows<2, 4, false>), grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace ac
