// Parts shared by the operators' kernels on the direct-to-LDS tile: 16-bit
// rows eight at a time, the epilogue slab, products with two segments of K,
// partial sums. Included INSIDE the kernels' namespace (an unnamed one in it),
// after dl_pipeline.h.

// Eight 16-bit values of a row from column c on; those at or past n are not
// touched (read as zero).
__device__ __forceinline__ u32x4 get8(const uint16_t* row, int64_t c, int64_t n) {
  if (c + 8 <= n) return load16(row + c);
  return load_row(row, c, n);
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

__device__ __forceinline__ void put8f(float* row, int64_t c, int64_t n, const float (&f)[8]) {
  if (c + 8 <= n) {
    const f32x4 lo = {f[0], f[1], f[2], f[3]}, hi = {f[4], f[5], f[6], f[7]};
    __builtin_memcpy(row + c, &lo, 16);
    __builtin_memcpy(row + c + 4, &hi, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) row[c + e] = f[e];
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
  __device__ __forceinline__ void add(int row, int c, f32x4 v) const {
    f32x4* at = reinterpret_cast<f32x4*>(p + row * (W * 4) + ((c ^ (row & (CH - 1))) << 4));
    *at += v;
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

__device__ __forceinline__ const char* uniform_ptr(const char* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}

// ---- operand tiles of a product with an optional second segment of K
// A lane's loads of one k-block, of both operands in one array (loads 0 ..
// NIA - 1 of A, then B's; RA, RB: the operands' DlOp, NB loads of a kind of
// B). As two DlOpTile members they kept the arrays of tiles whose operands are
// stored alike in scratch memory: before the loops over the loads are unrolled
// the compiler turns the branch between the two into a select of addresses.
template <class G, class RA, class RB>
struct LoadPlan {
  static constexpr int NL = G::NIA + RB::NI;
  int32_t off[NL];  // byte offset of the 16-byte chunk (OOB_OFF: outside)
  int32_t k[NL];    // its k within the block (where k runs along the stored rows)
  int32_t ka, kb;   // k-row of load 0 (where it does not)
  const char* baseA;
  const char* baseB;
  int64_t stepA, stepB;  // bytes from one k to the next
  int w;

  __device__ __forceinline__ void init(const uint16_t* A, int64_t lda, int64_t m0, int64_t left_a, const uint16_t* B,
                                       int64_t ldb, int64_t n0, int64_t left_b) {
    w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    DlOpTile<RA, G::BK> a;
    DlOpTile<RB, G::BK> b;
    a.init(A, lda, m0, left_a, w);
    b.init(B, ldb, n0, left_b, w);
#pragma unroll
    for (int q = 0; q < G::NIA; ++q) {
      off[q] = a.off[q];
      k[q] = RA::KC ? a.k[RA::KC ? q : 0] : 0;
    }
#pragma unroll
    for (int q = 0; q < RB::NI; ++q) {
      off[G::NIA + q] = b.off[q];
      k[G::NIA + q] = RB::KC ? b.k[RB::KC ? q : 0] : 0;
    }
    ka = a.k[0];
    kb = b.k[0];
    baseA = a.base;
    baseB = b.base;
    stepA = a.kstep;
    stepB = b.kstep;
  }
  __device__ __forceinline__ void load(const char* cur, int32_t o, bool in, char* dst) const {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(cur), (short)0,
                                                                       (int)0x7FFFFFF0, (int)RSRC_WORD3);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 16, in ? o : OOB_OFF, 0, 0, 0);
  }
  // A's load q into its stage; cur: the block's first k, rem: k left from there
  __device__ __forceinline__ void load_a(const char* cur, int rem, char* stage, int q) const {
    const bool in = RA::KC ? k[q] < rem : ka < rem - (w * RA::NI + q) * RA::RPI;
    load(cur, off[q], in, stage + (w * RA::NI + q) * 1024);
  }
  __device__ __forceinline__ void load_b(const char* cur, int rem, char* stage, int q) const {
    const bool in = RB::KC ? k[G::NIA + q] < rem : kb < rem - (w * RB::NI + q) * RB::RPI;
    load(cur, off[G::NIA + q], in, stage + (w * RB::NI + q) * 1024);
  }
};

template <class G>
struct SegTile {
  LoadPlan<G, typename G::OA, typename G::OB> l;
  const char* a2;
  const char* b2;
  int64_t K;  // (of the register-load form, not used here)
  int kA, kB;    // k that a segment of each operand holds
  int seg, end;  // first k-block of the second segment, and past the partition

  __device__ __forceinline__ void init(const MultiProd& p, int64_t m0, int64_t n0, int kseg, int end_block) {
    l.init(p.A, p.lda, m0, p.eA - m0, p.B, p.ldb, n0, p.eB - n0);
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
    pa = (two ? t.a2 : t.l.baseA) + k * t.l.stepA;
    pb = (two ? t.b2 : t.l.baseB) + k * t.l.stepB;
    remA = blk < t.end ? t.kA - k : 0;
    remB = blk < t.end ? t.kB - k : 0;
  }
  __device__ __forceinline__ void next(const SegTile<G>& t) {
    ++blk;
    const bool two = blk == t.seg;
    pa = two ? t.a2 : pa + G::BK * t.l.stepA;
    pb = two ? t.b2 : pb + G::BK * t.l.stepB;
    remA = two ? t.kA : remA - G::BK;
    remB = two ? t.kB : remB - G::BK;
    if (blk >= t.end) remA = remB = 0;  // past the partition: zeros, no traffic
  }
  __device__ __forceinline__ void issue(const SegTile<G>& t, int q) const {
    if (q < G::NIA)
      t.l.load_a(pa, remA, sA, q);
    else
      t.l.load_b(pb, remB, sB, q - G::NIA);
  }
};

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
