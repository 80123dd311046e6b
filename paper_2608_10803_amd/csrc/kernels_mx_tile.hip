// gfx950 products of microscaled 4-bit matrices on a tile of LDS stages:
//   k_mx_tile        out = A B^T + bias; gated: act(A B^T) * (A B2^T), the tile's
//                    columns BN/2 rows of B and the same of B2, a wave's fragments
//                    alternating between them (as k_gated in kernels_ffn.hip);
//                    or the sums of a part of K
//   k_mx_sum         adds the parts in their order and does what the tile's
//                    epilogue would have
//
// A stage is 256 values of K: 128 bytes of codes a row, as 64 of a 16-bit matrix
// are, loaded by the same direct-to-LDS loads into the same swizzled slots
// (dl_pipeline.h), and eight scale bytes a row. v_mfma_scale_f32_32x32x64 takes a
// block of 32 values, 16 bytes, of a row a lane, and one byte of a register as its
// scale. A sum's order is free, so lanes 0-31 take the stage's blocks 0 .. 3 in its
// four instructions and lanes 32-63 blocks 4 .. 7, of both operands: a lane's four
// scales are then one dword of the row's scale bytes, read once a stage; the
// instruction's selector picks the byte. The scales come stage by stage, eight bytes
// a row (k_mx_prepare): eight bytes of each of 512 rows where they lie in the operands
// fetch 512 cache lines a stage, as many bytes as the codes (8192^3: 316 us against
// 277).
//
// The matrix instruction does four times the operations of the 16-bit one on the
// same bytes in the same time, so LDS, the caches and the pipeline see what they see
// of a 16-bit product of a quarter of the depth. 4096 x 14336 x 4096: 140 us (3.4
// PFLOP/s; the matrix cores busy half of it), of a 128 x 256 tile's 32500 clocks 5000
// until its first stage has come, 21500 in the loop (16400 of matrix instructions) and
// 5700 for its outputs; 8192 x 8192 x 32768 reaches 4.8 PFLOP/s on 256 x 256 tiles.
// So a third of a tile's clocks are its first loads and its outputs, and the clocks are
// slow: 1.6 GHz in this product, 1.5 at 8192^3 (matrix cores busy 0.67 of it), 2.1 in
// kernels that only move memory. Workgroups that stay and load the next tile's first
// stages under this one's outputs took 2 % less time for 10 % fewer clocks, so that it
// seems to be the card's power that sets them (it was not read), and 128-deep stages with
// two workgroups a CU 20 % more time. fp32 outputs: 167 us. Gated, 2048 x 14336 x 4096:
// 134 us with SiLU, 156 with the GELU of tanh, 184 with that of erf.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernel_args.h"
#include "ops.h"

#define AC_INPUT_F16 0
#ifndef AC_MX_PART
#define AC_MX_PART 0
#endif

namespace ac {

#include "device_common.h"

namespace {

#include "dl_pipeline.h"
#include "tile_ops.h"
#include "activations.h"

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight outputs of a row from column c on, as out_type.
__device__ __forceinline__ void put_out8(void* out, int64_t at, int64_t c, int64_t n, const float (&v)[8], int type) {
  if (type == AC_TYPE_F32) {
    put8f(static_cast<float*>(out) + at, c, n, v);
    return;
  }
  u32x4 h;
  if (type == AC_TYPE_BF16) {
    h = pack8(v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      h[e] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[2 * e]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[2 * e + 1]) << 16);
  }
  put8(static_cast<uint16_t*>(out) + at, c, n, h);
}
__device__ __forceinline__ void add_bias8(const float* bias, int64_t c, int64_t n, float (&v)[8]) {
  if (!bias) return;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < n) v[e] += bias[c + e];
}

// Eight 16-bit values of a lane that holds columns c + 4 hi .. + 3 (v[0 .. 3]) and c
// + 8 + 4 hi .. + 3 of a row, hi the lane's half of the wave, the other half the rest
// of the 16: the halves change (v_permlane32_swap), so that the lower one has the
// first eight columns and the upper one the last.
template <int T>
__device__ __forceinline__ u32x4 pack_swapped(const float (&v)[8]) {
  u32x4 o;
  if constexpr (T == AC_TYPE_BF16) {
    o = pack8(v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[2 * e]) |
             ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[2 * e + 1]) << 16);
  }
  const auto x = __builtin_amdgcn_permlane32_swap(o[0], o[2], false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(o[1], o[3], false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}

// The tile's traits: codes as 16-bit units, 64 of them a stage and row.
template <int BM, int BN, int S, bool GATED>
struct Mx : Dl<BM, BN, 64, S, 2> {
  typedef Dl<BM, BN, 64, S, 2> D;
  typedef DlOp<GATED ? BN / 2 : BN, 64, true> OH;
  static constexpr int HALF = OH::BYTES;
  // a stage's scales: 128 rows, 1 KB, a load; A's, B's and (gated) B2's, a load a wave
  static constexpr int SA = (BM + 127) / 128, SB = (OH::EXT + 127) / 128;
  static constexpr int S_BYTES = 4096;
  static constexpr int LOADS = D::LOADS + 1;
  static_assert(SA + SB * (GATED ? 2 : 1) <= 4, "one load a wave");
  static constexpr int LDS = S * ((BM + BN) * 128 + S_BYTES);
  static constexpr int WPE = LDS <= 80 * 1024 && BM * BN <= 256 * 128 ? 2 : 1;
  static_assert(LDS <= 160 * 1024 && (!GATED || D::TN % 2 == 0), "tile");
};

template <class G>
struct MxPlan {
  LoadPlan<G, typename G::OA, typename G::OH> l;
  const char* up;
  const char* scales;  // the wave's 128 rows of the first stage's scales (uniform)
  int64_t sstep;       // bytes from a stage's scales to the next one's
  int32_t soff;        // of the lane's two rows, or OOB_OFF
  int64_t units;       // 16-bit units of a row's codes
  template <bool GATED>
  __device__ __forceinline__ void init(const MxTileArgs& g, int64_t m0, int64_t n0) {
    const MxProduct& p = g.p;
    l.init(reinterpret_cast<const uint16_t*>(p.a.codes), p.a.ld / 2, m0, p.M - m0,
           reinterpret_cast<const uint16_t*>(p.b.codes), p.b.ld / 2, n0, p.N - n0);
    up = GATED ? reinterpret_cast<const char*>(p.b2.codes + n0 * p.b.ld) : nullptr;
    units = (int64_t)p.blocks * 8;
    const bool isA = l.w < G::SA, isB = l.w < G::SA + G::SB, none = l.w >= G::SA + G::SB * (GATED ? 2 : 1);
    const int first = 128 * (l.w - (isA ? 0 : isB ? G::SA : G::SA + G::SB));
    const int64_t row0 = (isA ? m0 : n0) + first, left = (isA ? p.M : p.N) - row0;
    const int row = 2 * (int)(threadIdx.x & 63);
    scales = uniform_ptr(reinterpret_cast<const char*>((isA ? g.sa : isB ? g.sb : g.sb2) + row0 * 8));
    sstep = (isA ? g.lda : g.ldb) * 8;
    soff = row < left && !none ? row * 8 : OOB_OFF;
  }
};

template <class G, bool GATED>
struct MxLoads {
  const char* pa;
  const char* pg;
  const char* pu;
  const char* ps;
  int rem;  // 16-bit units of codes from the stage's first on, to the end of the partition or row
  char* sA;
  char* sB;
  char* sS;
  __device__ __forceinline__ void start(const MxPlan<G>& t, int beg, int end) {
    pa = t.l.baseA + (int64_t)beg * 128;
    pg = t.l.baseB + (int64_t)beg * 128;
    pu = t.up + (GATED ? (int64_t)beg * 128 : 0);
    rem = (int)(min((int64_t)end * 64, t.units) - (int64_t)beg * 64);
    ps = t.scales + beg * t.sstep;
  }
  __device__ __forceinline__ void next(const MxPlan<G>& t) {
    pa += 128;
    pg += 128;
    if constexpr (GATED) pu += 128;
    ps += t.sstep;
    rem -= 64;
  }
  __device__ __forceinline__ void issue(const MxPlan<G>& t, int q) const {
    constexpr int NH = G::OH::NI, NB = G::NIB;
    if (q < G::NIA) {
      t.l.load_a(pa, rem, sA, q);
    } else if (q < G::NIA + NH) {
      t.l.load_b(pg, rem, sB, q - G::NIA);
    } else if (q < G::NIA + NB) {
      t.l.load_b(pu, rem, sB + G::HALF, q - G::NIA - NH);
    } else {
      t.l.load(ps, t.soff, rem > 0, sS + t.l.w * 1024);
    }
  }
};

// Byte offsets of a lane's fragments in a stage: of k-step ks the block
// 4 (lane / 32) + ks of row lane % 32.
template <class O>
struct MxFragAddr {
  int at[4];
  __device__ __forceinline__ void init(int e0) {
    const int l32 = threadIdx.x & 31, hi = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      at[ks] = (e0 + l32) * O::ROW + (((4 * hi + ks) ^ swz_a<64>(l32)) << 4);
      asm("" : "+v"(at[ks]));
    }
  }
  __device__ __forceinline__ u32x4 read(const char* st, int ks, int i) const {
    return *reinterpret_cast<const u32x4*>(st + at[ks] + 32 * i * O::ROW);
  }
};
template <class G, bool GATED>
struct MxAddrs {
  MxFragAddr<typename G::OA> a;
  MxFragAddr<typename G::OH> b;
  int sa, sb;  // of the scale dwords
  __device__ __forceinline__ void init(int wr, int wc) {
    const int l32 = threadIdx.x & 31, hi = (threadIdx.x >> 5) & 1;
    const int e0 = GATED ? wc * G::WTN / 2 : wc * G::WTN;
    a.init(wr * G::WTM);
    b.init(e0);
    sa = (wr * G::WTM + l32) * 8 + hi * 4;
    sb = (128 * G::SA + e0 + l32) * 8 + hi * 4;
    asm("" : "+v"(sa));
    asm("" : "+v"(sb));
  }
  __device__ __forceinline__ u32x4 read_b(const char* st, int ks, int j) const {
    return GATED ? b.read(st + (j & 1) * G::HALF, ks, j >> 1) : b.read(st, ks, j);
  }
  __device__ __forceinline__ uint32_t scale_a(const char* st, int i) const {
    return *reinterpret_cast<const uint32_t*>(st + sa + 32 * 8 * i);
  }
  __device__ __forceinline__ uint32_t scale_b(const char* st, int j) const {
    return *reinterpret_cast<const uint32_t*>(st + sb + 8 * (GATED ? (j & 1) * 128 * G::SB + 32 * (j >> 1) : 32 * j));
  }
};
template <class G>
struct MxScales {
  uint32_t a[G::TM], b[G::TN];
};

template <int KS>
__device__ __forceinline__ f32x16 mx_mfma32(u32x4 a, uint32_t sa, u32x4 b, uint32_t sb, f32x16 c) {
  const i32x8 va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, c, 4, 4, KS, (int)sa, KS, (int)sb);
}
template <class G, int KS>
__device__ __forceinline__ void mx_step(const Frags<G>& f, const MxScales<G>& s, f32x16 (&acc)[G::TM][G::TN]) {
#pragma unroll
  for (int i = 0; i < G::TM; ++i)
#pragma unroll
    for (int j = 0; j < G::TN; ++j)  // C^T: a lane holds a row of C
      acc[i][j] = mx_mfma32<KS>(f.b[j], s.b[j], f.a[i], s.a[i], acc[i][j]);
}

template <int BM, int BN, int S, bool GATED, bool PART>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(Mx<BM, BN, S, GATED>::WPE, Mx<BM, BN, S, GATED>::WPE)))
void k_mx_tile(MxTileArgs g) {
  typedef Mx<BM, BN, S, GATED> G;
  AC_DL_STAGES(G);
  (void)lA4, (void)lB4;
  __shared__ __attribute__((aligned(1024))) char lS0[G::S_BYTES];
  __shared__ __attribute__((aligned(1024))) char lS1[G::S_BYTES];
  __shared__ __attribute__((aligned(1024))) char lS2[G::S_BYTES];
  __shared__ __attribute__((aligned(1024))) char lS3[G::S_BYTES];
  const MxProduct& p = g.p;
  int tm, tn;
  tile_coords(xcd_remap(blockIdx.x, g.tiles_m * g.tiles_n), g.tiles_m, g.tiles_n, 1, tm, tn);
  tm = __builtin_amdgcn_readfirstlane(tm);
  tn = __builtin_amdgcn_readfirstlane(tn);
  constexpr int NW = GATED ? BN / 2 : BN;  // columns of the output
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * NW;
  const int stages = (p.blocks + 7) / 8;
  const int beg = min((int)blockIdx.y * g.kper, stages), end = min(beg + g.kper, stages), nk = end - beg;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / G::WN, wc = wave % G::WN;
  MxPlan<G> t;
  t.template init<GATED>(g, m0, n0);

  f32x16 acc[G::TM][G::TN];
#pragma unroll
  for (int i = 0; i < G::TM; ++i)
#pragma unroll
    for (int j = 0; j < G::TN; ++j) acc[i][j] = f32x16{};

  // The pipeline of dl_main_loop.inc: a block's fragments are read one k-step
  // ahead of their instructions, also across stages; the scales of a stage with
  // its first fragments.
  constexpr int KS = 4, NMF = G::TM * G::TN, RD = G::TM + G::TN;
  constexpr int LSTEPS = S == 2 ? 2 : KS;
  constexpr int LPS = (G::LOADS + LSTEPS - 1) / LSTEPS, REST = G::LOADS - LPS;
  auto stA = [&](auto ic) -> char* {
    constexpr int I = decltype(ic)::value;
    return I == 0 ? lA0 : I == 1 ? lA1 : I == 2 ? lA2 : lA3;
  };
  auto stB = [&](auto ic) -> char* {
    constexpr int I = decltype(ic)::value;
    return I == 0 ? lB0 : I == 1 ? lB1 : I == 2 ? lB2 : lB3;
  };
  auto stS = [&](auto ic) -> char* {
    constexpr int I = decltype(ic)::value;
    return I == 0 ? lS0 : I == 1 ? lS1 : I == 2 ? lS2 : lS3;
  };
  MxAddrs<G, GATED> at;
  at.init(wr, wc);
  Frags<G> f[2];
  MxScales<G> sc, sn;
  MxLoads<G, GATED> nxt;
  auto read_frags = [&](auto ic, int ks, Frags<G>& to) {
    const char *a = stA(ic), *b = stB(ic);
#pragma unroll
    for (int i = 0; i < G::TM; ++i) to.a[i] = at.a.read(a, ks, i);
#pragma unroll
    for (int j = 0; j < G::TN; ++j) to.b[j] = at.read_b(b, ks, j);
  };
  auto read_scales = [&](auto ic, MxScales<G>& to) {
    const char* s = stS(ic);
#pragma unroll
    for (int i = 0; i < G::TM; ++i) to.a[i] = at.scale_a(s, i);
#pragma unroll
    for (int j = 0; j < G::TN; ++j) to.b[j] = at.scale_b(s, j);
  };
  auto into = [&](auto ic) {
    nxt.sA = stA(ic);
    nxt.sB = stB(ic);
    nxt.sS = stS(ic);
  };
  if (nk > 0) {
    nxt.start(t, beg, end);
    auto pro = [&](auto ic) {
      constexpr int I = decltype(ic)::value;
      if constexpr (I < S) {
        if (I > 0) nxt.next(t);
        into(ic);
#pragma unroll
        for (int q = 0; q < (I == S - 1 ? LPS : G::LOADS); ++q) nxt.issue(t, q);
      }
    };
    pro(std::integral_constant<int, 0>{});
    pro(std::integral_constant<int, 1>{});
    pro(std::integral_constant<int, 2>{});
    pro(std::integral_constant<int, 3>{});
    stage_barrier<(S - 1) * G::LOADS - REST>();
    read_scales(std::integral_constant<int, 0>{}, sc);
    read_frags(std::integral_constant<int, 0>{}, 0, f[0]);
    __builtin_amdgcn_sched_barrier(0);
  }
  // k-steps 0 .. 2 of the stage I; MORE: the rest of the loads of the stage issued last
  auto head = [&](auto ic, auto more) {
    constexpr bool MORE = decltype(more)::value && REST > 0;
    if constexpr (MORE) into(std::integral_constant<int, (decltype(ic)::value + S - 1) % S>{});
    auto one = [&](auto kc) {
      constexpr int ks = decltype(kc)::value;
      read_frags(ic, ks + 1, f[(ks + 1) & 1]);
      mx_step<G, ks>(f[ks & 1], sc, acc);
      if constexpr (MORE) {
#pragma unroll
        for (int q = (ks + 1) * LPS; q < (ks + 2) * LPS && q < G::LOADS; ++q) nxt.issue(t, q);
        interleave_step<NMF, RD, LPS>();
      } else {
        interleave_step<NMF, RD, 0>();
      }
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
  };
  // the barrier and the last k-step of the stage I, with the first reads of the
  // next one and the first loads of the stage S later
  auto tail = [&](auto ic) {
    constexpr int I = decltype(ic)::value;
    const std::integral_constant<int, (I + 1) % S> nx{};
    stage_barrier<(S - 2) * G::LOADS>();
    nxt.next(t);
    into(ic);
    read_scales(nx, sn);
    read_frags(nx, 0, f[0]);
    mx_step<G, 3>(f[1], sc, acc);
#pragma unroll
    for (int q = 0; q < LPS; ++q) nxt.issue(t, q);
    interleave_step<NMF, 2 * RD, LPS>();
    sc = sn;
  };
  auto step = [&](auto ic) {
    head(ic, std::true_type{});
    tail(ic);
  };
  // the last stages (at most S, all loading or loaded): stage I of them
  auto last = [&](auto ic, int left) {
    constexpr int I = decltype(ic)::value;
    if constexpr (I < S) {
      if (I >= left) return;
      head(ic, std::integral_constant<bool, I == 0>{});
      if (I + 1 < left) {
        const std::integral_constant<int, (I + 1) % S> nx{};
        stage_barrier<(S - 2 - I > 0 ? S - 2 - I : 0) * G::LOADS>();
        read_scales(nx, sn);
        read_frags(nx, 0, f[0]);
      }
      mx_step<G, 3>(f[1], sc, acc);
      __builtin_amdgcn_sched_barrier(0);
      sc = sn;
    }
  };
  int kb = 0;
  for (; nk - kb > S; kb += S) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    if constexpr (S > 2) step(std::integral_constant<int, 2>{});
    if constexpr (S > 3) step(std::integral_constant<int, 3>{});
  }
  last(std::integral_constant<int, 0>{}, nk - kb);
  last(std::integral_constant<int, 1>{}, nk - kb);
  last(std::integral_constant<int, 2>{}, nk - kb);
  last(std::integral_constant<int, 3>{}, nk - kb);

  stage_barrier<0>();  // no wave reads the stages any more, no load into them is in flight
  // A lane holds, of row l32 of a fragment, columns 8 q + 4 hi .. + 3 for q = 0 ..
  // 3. Stores are fast where neighbouring lanes write neighbouring bytes (128 KB by a
  // workgroup, 4 rows of 256 bytes a store: 2200 clocks, 32 rows of 32 bytes: 8000),
  // so outputs change lanes in LDS: 16-bit ones all at once, as they leave; fp32 ones,
  // and both GELUs, fragment row by fragment row in a loop (the code of an epilogue is
  // fetched once a tile, and 70 KB of it, erf's, took longer than the stores; that of
  // tanh would be as short as SiLU's). On 256 x 256 tiles without a split of K 552 bytes a
  // lane (gated 304) lie in scratch memory here, none in the main loop.
  constexpr int WW = GATED ? G::WTN / 2 : G::WTN;  // a wave's columns
  const int l32 = lane & 31, hi = lane >> 5;
  const int64_t rbase = m0 + wr * G::WTM, cbase = n0 + wc * WW;
  if constexpr (PART) {
#pragma unroll
    for (int i = 0; i < G::TM; ++i) {
      const int64_t row = rbase + 32 * i + l32;
      float* to = g.part + ((int64_t)blockIdx.y * p.M + row) * g.ldp + cbase + 4 * hi;
      if (row < p.M) {
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = 32 * (GATED ? j >> 1 : j) + 8 * q;
            // (the pitch is a multiple of 8: chunks are whole)
            if (cbase + c + 4 * hi < p.N)
              *reinterpret_cast<f32x4*>(to + (GATED && (j & 1) ? g.part2 : 0) + c) =
                  f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          }
      }
    }
    return;
  }
  char* const mine = slab_of<G>(wave, lA0, lA1, lA2, lB0, lB1, lB2, lB3);
  constexpr int LPR = WW / 8;  // lanes per row
  const int64_t c = cbase + (lane % LPR) * 8;
  if (p.out_type != AC_TYPE_F32 && (!GATED || p.act == AC_ACT_SILU)) {
    constexpr int P = WW * 2;  // bytes of a row: chunk k of it at k ^ row
    static_assert(G::WTM * P <= G::B_BYTES && (S >= 4 || G::WTM * P <= G::A_BYTES), "a wave's outputs fit a stage");
    auto fill = [&](auto type, auto with_bias) {
#pragma unroll
      for (int j = 0; j < G::TN; j += GATED ? 2 : 1)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = 4 * (GATED ? j >> 1 : j) + 2 * h;  // first chunk of the 16 columns
          float bias[8];
          if constexpr (decltype(with_bias)::value) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bias[e] = p.bias[min(cbase + 8 * k + 8 * (e >> 2) + 4 * hi + (e & 3), p.N - 1)];
          }
#pragma unroll
          for (int i = 0; i < G::TM; ++i) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = acc[i][j][8 * h + e];
              if constexpr (GATED) v[e] = v[e] * sigmoid(v[e]) * acc[i][GATED ? j + 1 : j][8 * h + e];
              if constexpr (decltype(with_bias)::value) v[e] += bias[e];
            }
            *reinterpret_cast<u32x4*>(mine + (32 * i + l32) * P + (((k + hi) ^ (l32 & (LPR - 1))) << 4)) =
                pack_swapped<decltype(type)::value>(v);
          }
        }
    };
    const std::integral_constant<int, AC_TYPE_BF16> bf{};
    const std::integral_constant<int, AC_TYPE_F16> hf{};
    if (GATED || !p.bias) {
      if (p.out_type == AC_TYPE_BF16)
        fill(bf, std::false_type{});
      else
        fill(hf, std::false_type{});
    } else if constexpr (!GATED) {
      if (p.out_type == AC_TYPE_BF16)
        fill(bf, std::true_type{});
      else
        fill(hf, std::true_type{});
    }
    constexpr int RPP = 64 / LPR, PASSES = G::WTM / RPP, U = PASSES < 8 ? PASSES : 8;  // rows of a store, stores, in a batch
    const int r0 = lane / LPR;
    uint16_t* to = static_cast<uint16_t*>(p.out) + (rbase + r0) * p.ldo;
    const char* from = mine + r0 * P;
    const bool whole = n0 + NW <= p.N;
#pragma unroll 1
    for (int b = 0; b < PASSES; b += U) {
      u32x4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * RPP;  // (its place among LPR rows: the batch's first is a multiple of LPR)
        v[u] = *reinterpret_cast<const u32x4*>(from + u * RPP * P + (((lane % LPR) ^ (r & (LPR - 1))) << 4));
      }
      const int64_t row = rbase + r0 + b * RPP;
      if (whole) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (row + u * RPP < p.M) __builtin_memcpy(to + u * RPP * p.ldo + c, &v[u], 16);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (row + u * RPP < p.M) put8(to + u * RPP * p.ldo, c, p.N, v[u]);
      }
      to += U * RPP * p.ldo;
      from += U * RPP * P;
    }
    static_assert(PASSES % U == 0 && (U * RPP) % LPR == 0, "batches");
    return;
  }
  const Slab<G::WTN> s = {mine};
#pragma unroll
  for (int i = 0; i < G::TM; ++i) {
    slab_fill<G>(s, acc[i], [](int j) { return GATED ? (j & 1) * WW + 32 * (j >> 1) : 32 * j; });
#pragma unroll 1
    for (int r = lane / LPR; r < 32; r += 64 / LPR) {
      const int64_t row = rbase + 32 * i + r;
      float v[8];
      s.get(r, lane % LPR, v);
      if constexpr (GATED) {
        float u[8], a[8];
        s.get(r, LPR + lane % LPR, u);
        act8(p.act, v, a);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = a[e] * u[e];
      }
      if (row < p.M && c < p.N) {
        if constexpr (!GATED) add_bias8(p.bias, c, p.N, v);
        put_out8(p.out, row * p.ldo, c, p.N, v, p.out_type);
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // fragment row by fragment row: bounded live registers
  }
}

#if AC_MX_PART == 0
template <bool GATED>
__global__ __launch_bounds__(256) void k_mx_sum(MxTileArgs g) {
  const MxProduct& p = g.p;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= p.N) return;
  MultiProd m;
  m.M = p.M;
  m.ldp = g.ldp;
  for (int64_t row = blockIdx.y; row < p.M; row += gridDim.y) {
    float v[8];
    m.part = g.part;
    part_sum(m, g.pk, row, c, v);
    if constexpr (GATED) {
      float u[8], h[8];
      m.part = g.part + g.part2;
      part_sum(m, g.pk, row, c, u);
      act8(p.act, v, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = h[e] * u[e];
    } else {
      add_bias8(p.bias, c, p.N, v);
    }
    put_out8(p.out, row * p.ldo, c, p.N, v, p.out_type);
  }
}
#endif

}  // namespace

// ---- launchers, compiled in parts: a tile each
template <int BM, int BN, int S>
hipError_t launch_mx_tile_of(const MxTileArgs& g, bool gated, hipStream_t st) {
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n), (unsigned)g.pk), block(256);
  if (!gated) {
    if (g.pk > 1)
      hipLaunchKernelGGL((k_mx_tile<BM, BN, S, false, true>), grid, block, 0, st, g);
    else
      hipLaunchKernelGGL((k_mx_tile<BM, BN, S, false, false>), grid, block, 0, st, g);
    return hipGetLastError();
  }
  if constexpr (Dl<BM, BN, 64, S, 2>::TN % 2 == 0) {
    if (g.pk > 1)
      hipLaunchKernelGGL((k_mx_tile<BM, BN, S, true, true>), grid, block, 0, st, g);
    else
      hipLaunchKernelGGL((k_mx_tile<BM, BN, S, true, false>), grid, block, 0, st, g);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}
#define MX_TILE(a, b, c) template hipError_t launch_mx_tile_of<a, b, c>(const MxTileArgs&, bool, hipStream_t);
#if AC_MX_PART == 1
MX_TILE(256, 256, 2)
#elif AC_MX_PART == 2
MX_TILE(128, 256, 3)
#elif AC_MX_PART == 3
MX_TILE(128, 128, 2)
#elif AC_MX_PART == 4
MX_TILE(64, 256, 3)
MX_TILE(32, 128, 3)
#else
extern MX_TILE(256, 256, 2) extern MX_TILE(128, 256, 3) extern MX_TILE(128, 128, 2) extern MX_TILE(64, 256, 3)
extern MX_TILE(32, 128, 3)

hipError_t launch_mx_tile(const FfnTile& t, const MxTileArgs& g, bool gated, hipStream_t st) {
  if (g.pk < 1 || g.kper < 1 || (int64_t)g.kper * g.pk * 8 < g.p.blocks || (g.pk > 1 && !g.part))
    return hipErrorInvalidValue;
  const auto is = [&](int bm, int bn, int stages) { return t.bm == bm && t.bn == bn && t.stages == stages; };
  if (is(256, 256, 2)) return launch_mx_tile_of<256, 256, 2>(g, gated, st);
  if (is(128, 256, 3)) return launch_mx_tile_of<128, 256, 3>(g, gated, st);
  if (is(128, 128, 2)) return launch_mx_tile_of<128, 128, 2>(g, gated, st);
  if (is(64, 256, 3)) return launch_mx_tile_of<64, 256, 3>(g, gated, st);
  if (is(32, 128, 3)) return launch_mx_tile_of<32, 128, 3>(g, gated, st);
  return hipErrorInvalidValue;
}
hipError_t launch_mx_sum(const MxTileArgs& g, bool gated, hipStream_t st) {
  const dim3 grid((unsigned)((g.p.N + 2047) / 2048), (unsigned)(g.p.M < 32768 ? g.p.M : 32768));
  if (gated)
    hipLaunchKernelGGL((k_mx_sum<true>), grid, dim3(256), 0, st, g);
  else
    hipLaunchKernelGGL((k_mx_sum<false>), grid, dim3(256), 0, st, g);
  return hipGetLastError();
}
#endif

}  // namespace ac
