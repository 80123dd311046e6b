// C entry points of the microscaled 4-bit matrices: checks, workspace, choice
// of kernels, launches.
#include <cmath>
#include <cstring>

#include "ops.h"
#include "ops_host.h"

namespace {

using namespace ac::host;

bool is_type(int32_t t) { return t == AC_TYPE_F32 || t == AC_TYPE_BF16 || t == AC_TYPE_F16; }
int64_t blocks_of(int64_t K) { return cdiv(K, 32); }

// codes and scales of a matrix of rows x (32 blocks)
adaptcore_status mx_check(const ac::MxMat& m, int64_t rows, int64_t blocks) {
  if (m.ld < std::max<int64_t>(1, 16 * blocks) || m.lds < std::max<int64_t>(1, blocks))
    return invalid("pitch of codes or scales smaller than the row");
  if (m.ld >= AC_MAX_LD || m.lds >= AC_MAX_LD) return invalid("pitches must be below 2^23");
  if (rows > 0 && blocks > 0 && (!m.codes || !m.scales)) return invalid("null pointer of codes or scales");
  return AC_OK;
}

struct MxCall {
  int64_t M, N, K;
  int32_t a_type;
  const void* A;  // values, where a_type is not AC_TYPE_MXFP4
  int64_t lda;
  ac::MxProduct p;
  bool gated;
};

adaptcore_status mx_size(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || M >= (1LL << 31) || N < 0 || N >= (1LL << 31) || K < 0 || K >= AC_MAX_LD)
    return invalid("M and N must be in [0, 2^31), K in [0, 2^23)");
  return AC_OK;
}

adaptcore_status check_call(MxCall* c) {
  adaptcore_status st = mx_size(c->M, c->N, c->K);
  if (st != AC_OK) return st;
  if (c->a_type != AC_TYPE_MXFP4 && !is_type(c->a_type)) return unsupported("unknown type of A");
  if (!is_type(c->p.out_type)) return unsupported("unknown output type");
  const int64_t blocks = blocks_of(c->K);
  c->p.blocks = (int)blocks;
  c->p.M = c->M;
  c->p.N = c->N;
  if (c->a_type == AC_TYPE_MXFP4) {
    st = mx_check(c->p.a, c->M, blocks);
  } else {
    if (c->lda < std::max<int64_t>(1, c->K)) st = invalid("row pitch smaller than the row");
    else if (c->lda >= AC_MAX_LD) st = invalid("pitches must be below 2^23");
    else if (c->M > 0 && c->K > 0 && !c->A) st = invalid("null matrix pointer");
    else if (misaligned(c->A, type_bytes(c->a_type))) st = invalid("pointer not aligned to its element size");
  }
  if (st == AC_OK) st = mx_check(c->p.b, c->N, blocks);
  if (st == AC_OK && c->gated) st = mx_check(c->p.b2, c->N, blocks);
  if (st != AC_OK) return st;
  if (c->p.ldo < std::max<int64_t>(1, c->N)) return invalid("row pitch smaller than the row");
  if (c->p.ldo >= AC_MAX_LD) return invalid("pitches must be below 2^23");
  if (c->M > 0 && c->N > 0 && !c->p.out) return invalid("null matrix pointer");
  if (misaligned(c->p.out, type_bytes(c->p.out_type)) || misaligned(c->p.bias, 4))
    return invalid("pointer not aligned to its element size");
  return AC_OK;
}

// ---- how a product runs
// On tiles, us: L + rounds of the grid's workgroups (256, or 512 of the tiles that
// share a CU) of F + T a stage, + o for every 10^6 outputs; split in pk parts of K
// instead s1 + s2 for every 10^6 sums, which are written and read. Fitted to the times
// of 3061 configurations of 210 sizes (M 33 to 4096, N 512 to 14336, K 640 to 14336,
// plain and gated, 16-bit outputs and SiLU); of those sizes the chosen one is 0.8 %
// slower than the fastest on average, at worst 17 %. (GELU and fp32 outputs have another
// epilogue, 4096 x 14336 x 4096 167 us instead of 143, which no term stands for.)
struct MxTileCost {
  ac::FfnTile tile;
  bool gated, two;  // exists gated; two to a CU
  double L, F, T, s1, s2, o;
  double F1, T1;  // two: alone on its CU
};
constexpr MxTileCost kMxTiles[] = {
    {{256, 256, 2}, true, false, 2.76, 8.38, 1.016, 2.31, 1.332, 0.831, 0, 0},
    {{128, 256, 3}, true, false, 3.85, 1.75, 0.573, 4.15, 1.778, 1.095, 0, 0},
    {{128, 128, 2}, true, true, 3.04, 0.0, 0.902, 4.13, 1.636, 0.694, 0.0, 0.637},
    {{64, 256, 3}, true, false, 3.48, 0.57, 0.436, 3.54, 2.103, 1.175, 0, 0},
    {{32, 128, 3}, false, true, 2.83, 0.65, 0.470, 2.73, 2.220, 0.634, 0.39, 0.265},
};
constexpr double MX_PREPARE = 3.0;  // a launch in front of the tiles that only their operands need
double tile_cost(const MxTileCost& c, int64_t groups, int kper, int pk, double outputs, bool gated) {
  double t = c.L;
  if (c.two) {
    const int64_t rest = groups % 512;
    t += (double)(groups / 512) * (c.F + c.T * kper);
    if (rest > 0) t += rest > 256 ? c.F + c.T * kper : c.F1 + c.T1 * kper;
  } else {
    t += (double)cdiv(groups, 256) * (c.F + c.T * kper);
  }
  return t + (pk > 1 ? c.s1 + c.s2 * 1e-6 * outputs * pk * (gated ? 2 : 1) : c.o * 1e-6 * outputs);
}
// On k_mx_rows, the same way (16 rows of B and 32 of A a workgroup, a stage of 512 k
// a wave of four; values: A quantised into the lanes' order first). Of 135 sizes (M 33
// to 512) the faster of rows and tiles is missed by 0.3 % on average, at worst by 9 %.
double rows_cost(int64_t M, int64_t N, int64_t blocks, bool gated, bool values) {
  const double groups = std::max(1.0, (double)(cdiv(N, 16) * cdiv(M, 32)) / 256.0), stages = (double)cdiv(cdiv(blocks, 16), 4);
  if (values) return gated ? 2.09 + groups * (1.26 * stages - 0.16) : 2.28 + groups * (0.66 * stages - 0.09);
  return gated ? 1.42 + groups * (0.52 + 1.79 * stages) : 1.56 + groups * (1.16 + 0.90 * stages);
}

struct MxWay {
  bool rows;
  bool fused;  // (rows) quantises A itself
  int waves;   // (rows)
  MxTileCost tile;
  int tiles_m, tiles_n, pk, kper;
};
constexpr int64_t MX_ROWS_MOST = 512;  // rows up to which k_mx_rows is asked
bool codes_direct(const ac::MxMat& m) {
  return (reinterpret_cast<uintptr_t>(m.codes) & 15) == 0 && m.ld % 16 == 0;
}
// values: A is quantised by the call; b_direct: B's codes lie as tiles load them.
adaptcore_status mx_way(int64_t M, int64_t N, int64_t K, bool gated, bool values, bool b_direct, MxWay* w) {
  const int64_t blocks = blocks_of(K);
  const int stages = (int)cdiv(blocks, 8);
  std::memset(w, 0, sizeof *w);
  double best = INFINITY;
  // (Up to 32 rows nothing is asked: of 9 shapes from 1024 x 1024 to 14336 x 4096, plain
  // and gated, codes and values, rows took 2.4 to 18.8 us, tiles and the launch in front
  // 5.9 to 25, but for codes of 17 to 32 rows with 14336 x 4096: 12.9 to 14.2 us against
  // 12.0, gated 17.8 to 18.8 against 17.3.)
  w->rows = M <= 32 || stages < 1;
  for (const MxTileCost& c : kMxTiles) {
    if ((gated && !c.gated) || w->rows) continue;
    const int64_t tm = cdiv(M, c.tile.bm), tn = cdiv(N, gated ? c.tile.bn / 2 : c.tile.bn), tiles = tm * tn;
    if (tm >= (1 << 30) || tn >= (1 << 30) || tiles >= (1LL << 31) / 256) continue;
    for (int pk : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      const int kper = (int)cdiv(stages, pk);
      if (pk > 1 && (kper < 2 || cdiv(stages, kper) != pk || tiles * pk > 1024)) continue;
      const double t = tile_cost(c, tiles * pk, kper, pk, (double)M * (double)N, gated);
      if (t < best) {
        best = t;
        w->tile = c;
        w->tiles_m = (int)tm;
        w->tiles_n = (int)tn;
        w->pk = pk;
        w->kper = kper;
      }
    }
  }
  // (codes that the tiles would copy first: 2 N K bytes less half, both ways)
  if (!b_direct) best += MX_PREPARE + 0.2e-6 * (double)N * (double)K * (gated ? 2 : 1);
  if (M <= MX_ROWS_MOST && !w->rows) w->rows = rows_cost(M, N, blocks, gated, values) <= best + (values ? 0 : MX_PREPARE);
  if (!w->rows && best == INFINITY) return unsupported("launch grid too large");
  if (w->rows) {
    // A quantised in the kernel costs every workgroup 0.4 us for each 4096 of its
    // values, in a launch of its own 1.5: us with 1 and 4 rows of 4096 x 4096 4.0 and
    // 5.3 against 5.4 and 5.7, 6 rows 6.4 and 6.0; 1 and 2 rows of 4096 x 14336 8.8 and
    // 10.7 against 9.1 and 9.2; of 14336 x 4096 7.9 and 10.5 against 9.6 and 9.6. The
    // bound is a little high: of nine shapes, plain and gated, all 31 pairs up to 16000 are
    // faster this way, by 15 % on average, 12 of 18 from there to 20500, by 3, but 2 of 10
    // up to 28000, which lose 7, and 2 of 13 up to 33000, which would lose 16.
    w->fused = values && M <= 16 && M * K * cdiv(N, 4096) * (gated ? 2 : 1) <= 28000 &&
               ac::mx_rows_lds(M, blocks) <= ac::MX_ROWS_LDS;
    // eight waves where one workgroup a CU has work for them (368 sizes: 1 % slower than
    // the better of four and eight on average; four always 1 to 2, A quantised in the
    // kernel 11; eight always up to 17)
    w->waves = cdiv(N, 16) * cdiv(M, 32) <= 256 ? 8 : 4;
  }
  return AC_OK;
}

bool quantises(const MxCall& c) { return c.a_type != AC_TYPE_MXFP4 && c.K > 0; }
bool b_codes_direct(const MxCall& c) { return codes_direct(c.p.b) && (!c.gated || codes_direct(c.p.b2)); }

// Counts the workspace, or (s->base) launches. a_direct, b_direct: A's and B's codes can
// be loaded where they lie.
adaptcore_status run_mx(MxCall c, const MxWay& w, bool a_direct, bool b_direct, Scratch* s, hipStream_t st, int* launches) {
  const bool run = s->base != nullptr, values = quantises(c);
  const int64_t blocks = blocks_of(c.K), stages = cdiv(blocks, 8);
  hipError_t e = hipSuccess;
  ac::MxQuantArgs q = {c.A, c.lda, c.M, c.K, nullptr, 0, nullptr, 0, ac::MX_IN_ROWS};
  int n = 0;
  if (w.rows) {
    if (values && !w.fused) {
      const int64_t stages16 = cdiv(blocks, 16), tiles = c.M > 16 ? cdiv(c.M, 32) * 2 : 1;
      q.order = ac::MX_IN_LANES;
      q.lds = stages16;
      q.codes = s->take<uint8_t>(tiles * stages16 * 4096);
      q.scales = s->take<uint8_t>(tiles * stages16 * 256);
      c.p.a = {q.codes, q.ld, q.scales, q.lds};
      if (run) e = ac::launch_mx_quantize(q, c.a_type, false, st);
      ++n;
    }
    const bool direct = a_direct && b_direct;
    if (run && e == hipSuccess)
      e = ac::launch_mx_rows(c.p, c.gated, w.fused ? &q : nullptr, c.a_type, values && !w.fused, w.waves, direct, st);
    ++n;
  } else {
    ac::MxPrepare prep;
    std::memset(&prep, 0, sizeof prep);
    ac::MxTileArgs t;
    std::memset(&t, 0, sizeof t);
    t.lda = cdiv(c.M, 2) * 2;
    t.ldb = cdiv(c.N, 2) * 2;
    // the operand's scales stage by stage, its codes copied where they are misaligned
    // (both of a pair's, which are read at one pitch)
    auto move = [&](ac::MxMat* m, int64_t rows, int64_t ld, bool ok) {
      uint8_t* const to = s->take<uint8_t>(stages * ld * 8);
      prep.m[prep.n++] = {m->scales, m->lds, to, ld, rows, (int)blocks, true};
      if (!ok) {
        uint8_t* const codes = s->take<uint8_t>(rows * blocks * 16);
        prep.m[prep.n++] = {m->codes, m->ld, codes, blocks * 16, rows, (int)blocks * 16, false};
        m->codes = codes;
        m->ld = blocks * 16;
      }
      return to;
    };
    if (values) {
      q.ld = stages * 128;
      q.lds = t.lda;
      q.order = ac::MX_IN_STAGES;
      q.codes = s->take<uint8_t>(c.M * q.ld);
      q.scales = s->take<uint8_t>(stages * t.lda * 8);
      prep.q = q;
      c.p.a = {q.codes, q.ld, nullptr, 0};
      t.sa = q.scales;
    } else {
      t.sa = move(&c.p.a, c.M, t.lda, a_direct);
    }
    t.sb = move(&c.p.b, c.N, t.ldb, b_direct);
    if (c.gated) t.sb2 = move(&c.p.b2, c.N, t.ldb, b_direct);
    t.p = c.p;
    t.tiles_m = w.tiles_m;
    t.tiles_n = w.tiles_n;
    t.pk = w.pk;
    t.kper = w.kper;
    if (w.pk > 1) {
      t.ldp = up8(c.N);
      t.part2 = (int64_t)w.pk * c.M * t.ldp;
      t.part = s->take<float>(t.part2 * (c.gated ? 2 : 1));
    }
    if (run) {
      e = ac::launch_mx_prepare(prep, c.a_type, st, &n);
      if (e == hipSuccess) e = ac::launch_mx_tile(w.tile.tile, t, c.gated, st);
      if (e == hipSuccess && w.pk > 1) e = ac::launch_mx_sum(t, c.gated, st);
      n += w.pk > 1 ? 2 : 1;
    }
  }
  *launches += n;
  if (e == hipErrorInvalidValue) return unsupported("launch grid too large");
  return launched(e, 0);
}

adaptcore_status product(MxCall c, hipStream_t s) {
  adaptcore_status st = check_call(&c);
  if (st != AC_OK || c.M == 0 || c.N == 0) return st;
  st = ac::op_ready();
  if (st != AC_OK) return st;
  const bool b_direct = b_codes_direct(c), a_direct = quantises(c) || codes_direct(c.p.a);
  MxWay way;
  st = mx_way(c.M, c.N, c.K, c.gated, quantises(c), b_direct, &way);
  if (st != AC_OK) return st;
  return with_scratch(s, [&](Scratch* w, int* n) { return run_mx(c, way, a_direct, b_direct, w, s, n); });
}

}  // namespace

extern "C" {

adaptcore_status adaptcore_mxfp4_quantize(int64_t rows, int64_t cols, int32_t type, uint32_t layout, const void* X,
                                          int64_t ldx, uint8_t* codes, int64_t ld_codes, uint8_t* scales,
                                          int64_t ld_scales, void* stream) {
  return guarded([&] {
    if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 30))
      return invalid("rows must be in [0, 2^31) and cols in [0, 2^30)");
    if (!is_type(type)) return unsupported("unknown element type");
    if (layout != AC_LAYOUT_ROW_ROW && layout != AC_LAYOUT_A_COL) return unsupported("unknown layout");
    const bool col = layout == AC_LAYOUT_A_COL;
    const int64_t blocks = blocks_of(cols);
    if (ldx < std::max<int64_t>(1, col ? rows : cols) || ld_codes < std::max<int64_t>(1, 16 * blocks) ||
        ld_scales < std::max<int64_t>(1, blocks))
      return invalid("row pitch smaller than the row");
    if (rows == 0 || cols == 0) return AC_OK;
    if (!X || !codes || !scales) return invalid("null pointer");
    if (misaligned(X, type_bytes(type))) return invalid("pointer not aligned to its element size");
    const adaptcore_status st = ac::op_ready();
    if (st != AC_OK) return st;
    const ac::MxQuantArgs a = {X, ldx, rows, cols, codes, ld_codes, scales, ld_scales, ac::MX_IN_ROWS};
    const hipError_t e = ac::launch_mx_quantize(a, type, col, static_cast<hipStream_t>(stream));
    if (e == hipErrorInvalidValue) return unsupported("launch grid too large");
    return launched(e, 1);
  });
}

adaptcore_status adaptcore_mxfp4_dequantize(int64_t rows, int64_t cols, int32_t type, const uint8_t* codes,
                                            int64_t ld_codes, const uint8_t* scales, int64_t ld_scales, void* Y,
                                            int64_t ldy, void* stream) {
  return guarded([&] {
    if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 30))
      return invalid("rows must be in [0, 2^31) and cols in [0, 2^30)");
    if (!is_type(type)) return unsupported("unknown element type");
    const int64_t blocks = blocks_of(cols);
    if (ldy < std::max<int64_t>(1, cols) || ld_codes < std::max<int64_t>(1, 16 * blocks) ||
        ld_scales < std::max<int64_t>(1, blocks))
      return invalid("row pitch smaller than the row");
    if (rows == 0 || cols == 0) return AC_OK;
    if (!Y || !codes || !scales) return invalid("null pointer");
    if (misaligned(Y, type_bytes(type))) return invalid("pointer not aligned to its element size");
    const adaptcore_status st = ac::op_ready();
    if (st != AC_OK) return st;
    const ac::MxDequantArgs a = {{codes, ld_codes, scales, ld_scales}, rows, cols, Y, ldy};
    const hipError_t e = ac::launch_mx_dequantize(a, type, static_cast<hipStream_t>(stream));
    if (e == hipErrorInvalidValue) return unsupported("launch grid too large");
    return launched(e, 1);
  });
}

adaptcore_status adaptcore_mxfp4_matmul(int64_t M, int64_t N, int64_t K, int32_t a_type, const void* A, int64_t lda,
                                        const uint8_t* A_scales, int64_t ld_a_scales, const uint8_t* B, int64_t ldb,
                                        const uint8_t* B_scales, int64_t ld_b_scales, const float* bias,
                                        int32_t out_type, void* Y, int64_t ldy, void* stream) {
  return guarded([&] {
    MxCall c = {M, N, K, a_type, A, lda, {}, false};
    c.p.a = {static_cast<const uint8_t*>(A), lda, A_scales, ld_a_scales};
    c.p.b = {B, ldb, B_scales, ld_b_scales};
    c.p.bias = bias;
    c.p.out = Y;
    c.p.ldo = ldy;
    c.p.out_type = out_type;
    return product(c, static_cast<hipStream_t>(stream));
  });
}

adaptcore_status adaptcore_mxfp4_gated_matmul(int64_t M, int64_t F, int64_t K, int32_t a_type, const void* A,
                                              int64_t lda, const uint8_t* A_scales, int64_t ld_a_scales,
                                              const uint8_t* Bg, const uint8_t* Bu, int64_t ldb,
                                              const uint8_t* Bg_scales, const uint8_t* Bu_scales, int64_t ld_b_scales,
                                              int32_t activation, int32_t type, void* H, int64_t ldh, void* stream) {
  return guarded([&] {
    if (activation != AC_ACT_SILU && activation != AC_ACT_GELU && activation != AC_ACT_GELU_TANH)
      return unsupported("unknown activation");
    MxCall c = {M, F, K, a_type, A, lda, {}, true};
    c.p.a = {static_cast<const uint8_t*>(A), lda, A_scales, ld_a_scales};
    c.p.b = {Bg, ldb, Bg_scales, ld_b_scales};
    c.p.b2 = {Bu, ldb, Bu_scales, ld_b_scales};
    c.p.out = H;
    c.p.ldo = ldh;
    c.p.out_type = type;
    c.p.act = activation;
    return product(c, static_cast<hipStream_t>(stream));
  });
}

int64_t adaptcore_mxfp4_workspace(int64_t M, int64_t N, int64_t K, int32_t gated) {
  int64_t bytes = 0;
  const adaptcore_status st = guarded([&] {
    adaptcore_status rc = mx_size(M, N, K);
    if (rc != AC_OK || M == 0 || N == 0) return rc;
    for (int32_t a_type : {AC_TYPE_MXFP4, (int)AC_TYPE_BF16})
      for (int bad = 0; bad < 4; ++bad) {
        MxCall c = {};
        c.M = M;
        c.N = N;
        c.K = K;
        c.a_type = a_type;
        c.gated = gated != 0;
        c.p.blocks = (int)blocks_of(K);
        Scratch s;
        int n = 0;
        const bool b_direct = !(bad & 2);
        MxWay way;
        rc = mx_way(M, N, K, c.gated, quantises(c), b_direct, &way);
        if (rc == AC_OK) rc = run_mx(c, way, quantises(c) || !(bad & 1), b_direct, &s, nullptr, &n);
        if (rc != AC_OK) return rc;
        bytes = std::max(bytes, s.used);
      }
    return AC_OK;
  });
  return st == AC_OK ? bytes : (int64_t)st;
}

adaptcore_status adaptcore_mxfp4_kernels(int64_t M, int64_t N, int64_t K, int32_t gated, int32_t a_type, char* buf,
                                         int64_t len) {
  return guarded([&] {
    if (!buf || len < 1) return invalid("null argument");
    const adaptcore_status rc = mx_size(M, N, K);
    if (rc != AC_OK) return rc;
    if (a_type != AC_TYPE_MXFP4 && !is_type(a_type)) return unsupported("unknown type of A");
    std::string out;
    if (M > 0 && N > 0) {
      const bool values = a_type != AC_TYPE_MXFP4 && K > 0;
      MxWay w;
      const adaptcore_status r2 = mx_way(M, N, K, gated != 0, values, true, &w);
      if (r2 != AC_OK) return r2;
      if (w.rows) {
        out = std::string(values && !w.fused ? "k_mx_quant;" : "") + "k_mx_rows<" + std::to_string(M > 16 ? 2 : 1) + ">";
      } else {
        out = "k_mx_prepare;k_mx_tile<" + std::to_string(w.tile.tile.bm) + ", " + std::to_string(w.tile.tile.bn) + ">";
        if (w.pk > 1) out += " x" + std::to_string(w.pk) + ";k_mx_sum";
      }
    }
    if ((int64_t)out.size() + 1 > len) return invalid("buffer too small");
    std::memcpy(buf, out.c_str(), out.size() + 1);
    return AC_OK;
  });
}

}  // extern "C"
