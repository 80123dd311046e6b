// The direct-to-LDS tile's parts shared by the kernel files that multiply on
// it: operand tiles loaded straight into LDS stages and MFMA fragment reads.
// What they do and why is at the head of kernels_dl.hip; the main loop over
// them is dl_main_loop.inc. Included INSIDE the kernels' namespace (an unnamed
// one in it), after device_common.h.

// the transpose read moves 16-bit patterns; its bf16 form serves fp16 too
typedef __bf16 tr16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) tr16x4 lds_tr16x4;

enum DlOut : int { DL_F32 = 0, DL_BF16 = 1, DL_PARTIAL = 2 };

// One operand's tile of a stage: EXT rows of A (or columns of B) by BK of k.
// KC: k runs along the stored rows (a row-major A, a column-major B): EXT rows
// of BK, MFMA fragments read with ds_read_b128. Otherwise the extent does (a
// row-major B, a column-major A): BK rows of EXT, fragments read with the
// transpose read. Either way 16-byte chunks swizzled within their row, and a
// lane gets the same 8 consecutive k of the same row or column.
template <int EXT_, int BK, bool KC_>
struct DlOp {
  static constexpr int EXT = EXT_;
  static constexpr bool KC = KC_;
  static constexpr int ROW = (KC ? BK : EXT) * 2;  // bytes of a stored row
  static constexpr int BYTES = EXT * BK * 2;
  static constexpr int LPR = ROW / 16;     // 16-byte chunks of a row
  static constexpr int RPI = 64 / LPR;     // rows per wave-wide load
  static constexpr int NI = BYTES / 4096;  // wave-wide loads per wave and stage
  static constexpr int READS = KC ? 1 : 2; // LDS reads of a fragment
  static_assert(KC || EXT >= 128, "the k-row swizzle spans 16 chunks");
};

// LAY: bit 0, A column-major in memory; bit 1, B column-major.
template <int BM, int BN, int BK_, int S_, int LAY = 0>
struct Dl {
  static constexpr int BN_ = BN, BK = BK_, S = S_, NT = 256;
  // waves: 2 x 2 quadrants, or (tiles of at most 64 rows: the decode-style
  // shapes) 1 x 4 along N
  static constexpr int WM = BM >= 128 ? 2 : 1, WN = 4 / WM;
  static constexpr int WTM = BM / WM, WTN = BN / WN;  // a wave's part of the tile
  static constexpr int TM = WTM / 32, TN = WTN / 32;
  typedef DlOp<BM, BK, (LAY & 1) == 0> OA;
  typedef DlOp<BN, BK, (LAY & 2) != 0> OB;
  static constexpr int A_BYTES = OA::BYTES, B_BYTES = OB::BYTES;
  static constexpr int A_LPR = OA::LPR, A_RPI = OA::RPI, B_LPR = OB::LPR, B_RPI = OB::RPI;
  static constexpr int NIA = OA::NI, NIB = OB::NI;
  static constexpr int LOADS = NIA + NIB;
  static constexpr int CT_LD = WTN + 4;       // padded row of the bf16 output slab
  // workgroups per CU the configuration is built for: two when two fit the
  // LDS and the register file (two waves per SIMD, at most 256 registers
  // each): one workgroup's epilogue stores then overlap the other's loads
  // and MFMAs
  static constexpr int WPE = (S * (BM + BN) * BK * 2 <= 80 * 1024 && BM * BN <= 256 * 128) ? 2 : 1;
  static_assert(BM % 32 == 0 && BM >= 32 && BN >= 128 && BN <= 512 && (BK == 32 || BK == 64) && WTN % 32 == 0,
                "tile");
  // the bf16 epilogue's per-wave slab of 32 output rows goes into one stage
  // buffer per wave: A0, A1, B0, B1 if both kinds are large enough, else
  // the first four of the kind that is, else two slabs in each of B0, B1
  static constexpr int SLAB = 32 * CT_LD * 2;
  static constexpr int SLAB_KIND = (SLAB <= A_BYTES && SLAB <= B_BYTES) ? 0
                                   : (SLAB <= B_BYTES && S >= 4)        ? 1
                                   : (2 * SLAB <= B_BYTES)              ? 3
                                                                        : 2;
  static_assert(SLAB_KIND != 2 || (SLAB <= A_BYTES && S >= 4), "output slab fits a stage buffer");
};

// B stage: chunk c of k-row r sits at slot c ^ f(r & 3), f = 0, 6, 12, 10.
// One transpose read covers 4 consecutive k-rows and 2 (16 lanes) or 4 (32
// lanes) consecutive chunks; f keeps those on distinct banks for both 32
// and 64 banks.
__device__ __forceinline__ int swz_b(int r) { return (0xAC60 >> (4 * (r & 3))) & 15; }

// Workgroup barrier of the pipeline: this wave waits until at most N of its
// loads into LDS are in flight and its own LDS reads and writes are done,
// then all waves meet. After it every wave's older loads have landed and no
// wave still reads what it read before. (__syncthreads would add a workgroup
// fence, which waits for ALL loads into LDS, the prefetched stages included.)
// The empty asm with a memory clobber keeps the compiler from moving LDS
// accesses across it.
template <int N>
__device__ __forceinline__ void stage_barrier() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(N));
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Addressing of a workgroup's loads of one operand: the byte offset of every
// 16-byte chunk this lane loads (OOB_OFF for rows and columns outside the
// matrix), and the k of that chunk within the block for the K tail.
template <class O, int BK>
struct DlOpTile {
  const char* base;       // the tile's first row (column) at k = 0
  int64_t kstep;          // bytes from one k to the next
  int32_t off[O::NI];
  int32_t k[O::KC ? O::NI : 1];  // KC: k of each chunk; else the k-row of the first one

  // p: the operand, ld its row pitch, e0 the tile's first row or column, left
  // how many of them the matrix has from there on
  __device__ __forceinline__ void init(const uint16_t* p, int64_t ld, int64_t e0, int64_t left, int w) {
    const int lane = threadIdx.x & 63;
    base = reinterpret_cast<const char*>(p + e0 * (O::KC ? ld : 1));
    kstep = 2 * (O::KC ? 1 : ld);
    if constexpr (!O::KC) k[0] = lane / O::LPR;
#pragma unroll
    for (int q = 0; q < O::NI; ++q) {
      const int row = (w * O::NI + q) * O::RPI + lane / O::LPR;  // stored row of the tile
      const int c = (lane % O::LPR) ^ (O::KC ? swz_a<BK>(row) : swz_b(row));  // the chunk this slot holds
      off[q] = (O::KC ? row : c * 8) < left ? (int32_t)(row * ld * 2) + c * 16 : OOB_OFF;
      if constexpr (O::KC) k[q] = c * 8;
    }
  }
  // load q (a compile-time index) of wave w into a stage: cur = the block's
  // first k, rem = k left from there
  __device__ __forceinline__ void issue(const char* cur, int rem, char* stage, int w, int q) const {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(cur), (short)0,
                                                                       (int)0x7FFFFFF0, (int)RSRC_WORD3);
    const bool in = O::KC ? k[O::KC ? q : 0] < rem : k[0] < rem - (w * O::NI + q) * O::RPI;
    const int32_t o = in ? off[q] : OOB_OFF;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(stage + (w * O::NI + q) * 1024), 16, o, 0, 0, 0);
  }
};

template <class G>
struct DlTile {
  DlOpTile<typename G::OA, G::BK> a;
  DlOpTile<typename G::OB, G::BK> b;
  int64_t K, kA, kB;  // k of the loop; k each operand holds
  int w;              // wave (uniform)

  __device__ __forceinline__ void init(const GemmArgs& g, int64_t m0, int64_t n0) {
    w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    K = g.K;
    // (g.K is rounded up to 8 when A is a zero-padded row-major copy)
    kA = G::OA::KC ? g.K : g.kB;
    kB = G::OB::KC ? g.K : g.kB;
    a.init(g.A, g.lda, m0, g.M - m0, w);
    b.init(g.B, g.ldb, n0, (G::OB::KC ? g.N : g.nB) - n0, w);
  }
};

// This wave's share of the loads of one k-block into one stage: NIA loads of
// A, then NIB loads of B, issued one at a time so that they can be spread
// between MFMAs. The blocks are taken in order from `kbeg` on; what a block
// has past the partition's end (the k tail, or a whole block past it) is out
// of range and read as zeros. A step to the next block is a few scalar
// additions: a wave issues one instruction at a time, and the MFMAs wait for
// whatever scalar work stands in front of them.
template <class G>
struct StageLoads {
  const char* pa;  // the block's first k of A's tile, and of B's
  const char* pb;
  int remA, remB;  // k of A and of B from there to the partition's end
  char* sA;
  char* sB;
  __device__ __forceinline__ void start(const DlTile<G>& t, int64_t kbeg, int64_t kstop) {
    pa = t.a.base + kbeg * t.a.kstep;
    pb = t.b.base + kbeg * t.b.kstep;
    remA = (int)(min(kstop, t.kA) - kbeg);
    remB = (int)(min(kstop, t.kB) - kbeg);
  }
  __device__ __forceinline__ void next(const DlTile<G>& t) {
    pa += G::BK * t.a.kstep;
    pb += G::BK * t.b.kstep;
    remA -= G::BK;
    remB -= G::BK;
  }
  // load q of this wave (0 .. NIA + NIB - 1; a compile-time index)
  __device__ __forceinline__ void issue(const DlTile<G>& t, int q) const {
    if (q < G::NIA)
      t.a.issue(pa, remA, sA, t.w, q);
    else
      t.b.issue(pb, remB, sB, t.w, q - G::NIA);
  }
};

// ---- loads through registers (any alignment, K >= 8 and N >= 8)
// The same chunks into the same LDS slots as the direct loads, fetched with
// 16-byte loads at any 2-byte address: a chunk that crosses the end of a
// row is loaded as the 16 bytes ending at the row end and shifted down in
// registers, with zeros past K (A columns, B rows) and past N (B columns).
// Rows past M re-read row M - 1 (their outputs are never stored).
template <class G>
struct DlTileU {
  const uint16_t* a;  // A + m0 * lda
  const uint16_t* B;
  int64_t ldb, K, N;
  uint32_t a_row[G::NIA];  // bytes: clamped row * lda * 2
  int32_t a_c[G::NIA];     // k of the chunk within the block
  int32_t b_kr[G::NIB];    // k-row of the chunk within the block
  uint32_t b_col[G::NIB];  // bytes: first column loaded (<= N - 8)
  int32_t b_cs[G::NIB];    // elements dropped at the N edge (0 .. 8)

  __device__ __forceinline__ void init(const GemmArgs& g, int64_t m0, int64_t n0) {
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    a = g.A + m0 * g.lda;
    B = g.B;
    ldb = g.ldb;
    K = g.K;
    N = g.N;
#pragma unroll
    for (int q = 0; q < G::NIA; ++q) {
      const int u = w * G::NIA + q;
      const int row = u * G::A_RPI + lane / G::A_LPR;
      const int c = (lane % G::A_LPR) ^ swz_a<G::BK>(row);
      a_row[q] = (uint32_t)((min(m0 + row, g.M - 1) - m0) * g.lda * 2);
      a_c[q] = c * 8;
    }
#pragma unroll
    for (int q = 0; q < G::NIB; ++q) {
      const int u = w * G::NIB + q;
      const int kr = u * G::B_RPI + lane / G::B_LPR;
      const int c = (lane % G::B_LPR) ^ swz_b(kr);
      const int64_t gn = n0 + c * 8, st = min(gn, g.N - 8);
      b_kr[q] = kr;
      b_col[q] = (uint32_t)(st * 2);
      b_cs[q] = (int32_t)min(gn - st, (int64_t)8);
    }
  }
};

template <class G>
struct RegLoads {
  u32x4 va[G::NIA], vb[G::NIB];
  uint32_t sha, shb;  // per chunk 4 bits: elements to drop (8 = all)
  const uint16_t* a0;  // A tile base at this block's k (elements: the chunk's start added per lane)
  const uint16_t* b0;  // B + min(k0, K - 1) * ldb
  int64_t k0, kb0;
  char* sA;
  char* sB;
  __device__ __forceinline__ void init(char* a_stage, char* b_stage, const DlTileU<G>& t, int64_t k) {
    k0 = k;
    kb0 = min(k, t.K - 1);
    b0 = t.B + kb0 * t.ldb;
    sA = a_stage;
    sB = b_stage;
    sha = shb = 0;
  }
  // global load q into registers (0 .. NIA + NIB - 1, a compile-time index)
  __device__ __forceinline__ void issue(const DlTileU<G>& t, int q) {
    if (q < G::NIA) {
      const int64_t e = k0 + t.a_c[q], st = min(e, t.K - 8);
      const uint32_t s = (uint32_t)min(e - st, (int64_t)8);
      va[q] = load16(reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(t.a) + t.a_row[q] + st * 2));
      sha |= s << (4 * q);
    } else {
      const int qb = q - G::NIA;
      const int64_t r = k0 + t.b_kr[qb];
      const int64_t rr = min(r, t.K - 1) - kb0;  // >= 0
      vb[qb] = load16(reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(b0) +
                                                         (uint32_t)(rr * t.ldb * 2) + t.b_col[qb]));
      const uint32_t s = r >= t.K ? 8u : (uint32_t)t.b_cs[qb];
      shb |= s << (4 * qb);
    }
  }
  // the shifted chunks into their LDS slots (after the loads landed)
  __device__ __forceinline__ void finish() {
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int q = 0; q < G::NIA; ++q)
      *reinterpret_cast<u32x4*>(sA + (w * G::NIA + q) * 1024 + lane * 16) = shift_down(va[q], (sha >> (4 * q)) & 15);
#pragma unroll
    for (int q = 0; q < G::NIB; ++q)
      *reinterpret_cast<u32x4*>(sB + (w * G::NIB + q) * 1024 + lane * 16) = shift_down(vb[q], (shb >> (4 * q)) & 15);
  }
};

// Byte offsets of a lane's fragment reads within a stage, computed once. KC:
// one per k-step (rows are ROW bytes apart, and the swizzle of row 32 i + l32
// is that of l32); else one per fragment (k-step and half are constant
// offsets: the swizzle only depends on the k-row mod 4). Opaque to the
// compiler: it may not take the sums apart into a chain of address steps, at
// whose end it no longer knows which stage is read and would wait for the
// loads into all of them.
template <class O, int BK, int T>
struct FragAddr {
  int at[O::KC ? BK / 16 : T];
  __device__ __forceinline__ void init(int e0) {  // e0: the wave's first row or column in the tile
    const int lane = threadIdx.x & 63;
    const int l32 = lane & 31, hi = lane >> 5, i16 = lane & 15, g = lane >> 4;
    if constexpr (O::KC) {
#pragma unroll
      for (int ks = 0; ks < BK / 16; ++ks) {
        const int ch = 2 * ks + hi;  // 8 consecutive k of the lane's k-group
        at[ks] = (e0 + l32) * O::ROW + ((ch ^ swz_a<BK>(l32)) << 4);
        asm("" : "+v"(at[ks]));
      }
    } else {
      // the transpose read of a 16-lane group covers 4 k-rows x 16 columns: lane
      // i16 addresses k-row i16 >> 2 and columns 4 * (i16 & 3) .. +3 and receives
      // column i16 of the 4 rows; groups 0 / 1 take columns 0-15 / 16-31 of the
      // fragment at the lane's k-group 0, groups 2 / 3 the same at k-group 1
      const int kr0 = 8 * (g >> 1) + (i16 >> 2);
#pragma unroll
      for (int j = 0; j < T; ++j) {
        const int col = e0 + 32 * j + 16 * (g & 1) + (i16 & 3) * 4;
        at[j] = kr0 * O::ROW + ((col >> 3) ^ swz_b(kr0)) * 16 + (col & 7) * 2;
        asm("" : "+v"(at[j]));
      }
    }
  }
  // fragment i of k-step ks (compile-time indices)
  __device__ __forceinline__ u32x4 read(const char* st, int ks, int i) const {
    if constexpr (O::KC) {
      return *reinterpret_cast<const u32x4*>(st + at[ks] + 32 * i * O::ROW);
    } else {
      uint32_t v[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const tr16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_tr16x4*)(st + at[i] + (16 * ks + 4 * h) * O::ROW));
        const uint64_t bits = __builtin_bit_cast(uint64_t, r);
        v[2 * h] = (uint32_t)bits;
        v[2 * h + 1] = (uint32_t)(bits >> 32);
      }
      return u32x4{v[0], v[1], v[2], v[3]};
    }
  }
};

// Fragments of one k-step (16 k) of a stage.
template <class G>
struct Frags {
  u32x4 a[G::TM], b[G::TN];
};

template <class G>
struct FragAddrs {
  FragAddr<typename G::OA, G::BK, G::TM> a;
  FragAddr<typename G::OB, G::BK, G::TN> b;
};

template <class G, class Addrs>
__device__ __forceinline__ void read_frags(const char* sA, const char* sB, int ks, const Addrs& at, Frags<G>& f) {
#pragma unroll
  for (int i = 0; i < G::TM; ++i) f.a[i] = at.a.read(sA, ks, i);
#pragma unroll
  for (int j = 0; j < G::TN; ++j) f.b[j] = at.b.read(sB, ks, j);
}

// What runs under the NMF MFMAs of one k-step: RD LDS reads (the next step's
// fragments), two to an MFMA from the first one on, and LD global loads one
// to an MFMA. A wave that stalls on a full LDS or load queue issues no MFMAs,
// so neither may leave in a burst.
template <int NMF, int RD, int LD>
__device__ __forceinline__ void interleave_step() {
  constexpr int RPM = 2 * NMF >= RD ? 2 : (RD + NMF - 1) / NMF, LPM = (LD + NMF - 1) / NMF;
#pragma unroll
  for (int m = 0; m < NMF; ++m) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                      // one MFMA
    if (m * RPM < RD) __builtin_amdgcn_sched_group_barrier(0x100, RPM, 0);  // LDS reads
    if ((m + 1) * LD / NMF > m * LD / NMF) __builtin_amdgcn_sched_group_barrier(0x020, LPM, 0);  // loads
  }
  __builtin_amdgcn_sched_barrier(0);
}

template <class G>
__device__ __forceinline__ void mfma_step(const Frags<G>& f, f32x16 (&acc)[G::TM][G::TN]) {
#pragma unroll
  for (int i = 0; i < G::TM; ++i)
#pragma unroll
    for (int j = 0; j < G::TN; ++j) acc[i][j] = mfma32(f.b[j], f.a[i], acc[i][j]);  // C^T: a lane holds a row of C
}

// The LDS stages of a workgroup (up to five; those a kernel's main loop does
// not name take no room).
#define AC_DL_STAGES(G)                                           \
  __shared__ __attribute__((aligned(1024))) char lA0[G::A_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lA1[G::A_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lA2[G::A_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lA3[G::A_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lA4[G::A_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lB0[G::B_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lB1[G::B_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lB2[G::B_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lB3[G::B_BYTES]; \
  __shared__ __attribute__((aligned(1024))) char lB4[G::B_BYTES]
