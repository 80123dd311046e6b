// C entry points of the operators beside the products: checks, workspace,
// launches.
#include "ops.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <new>
#include <tuple>

#include "planner.h"
#include "registry.h"

namespace {

// No exception leaves a C entry point.
template <class F>
adaptcore_status guarded(F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return AC_ERR_OUT_OF_MEMORY;
  } catch (...) {
    return AC_ERR_INTERNAL;
  }
}

adaptcore_status launched(hipError_t e, int n) {
  if (e != hipSuccess)
    return ac::op_fail(AC_ERR_LAUNCH, std::string("kernel launch failed: ") + hipGetErrorString(e));
  ac::op_count_launches(n);
  return AC_OK;
}

adaptcore_status invalid(const char* msg) { return ac::op_fail(AC_ERR_INVALID_VALUE, msg); }
adaptcore_status unsupported(const char* msg) { return ac::op_fail(AC_ERR_UNSUPPORTED, msg); }

int type_bytes(int32_t t) { return t == AC_TYPE_F32 ? 4 : 2; }
bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// ---- layer norm
adaptcore_status norm_size(int64_t rows, int64_t cols) {
  if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 30))
    return invalid("rows must be in [0, 2^31) and cols in [0, 2^30)");
  return AC_OK;
}
adaptcore_status norm_types(int32_t type, int32_t weight_type) {
  if (type != AC_TYPE_F32 && type != AC_TYPE_BF16 && type != AC_TYPE_F16) return unsupported("unknown element type");
  if (weight_type != AC_TYPE_F32 && weight_type != type)
    return unsupported("the weights must be fp32 or of the rows' type");
  return AC_OK;
}

// ---- gated feed-forward block
int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Hands out pieces of a workspace (256-byte aligned); without a base it only
// counts.
struct Scratch {
  char* base = nullptr;
  int64_t used = 0;
  template <class T>
  T* take(int64_t n) {
    char* p = base ? base + used : nullptr;
    used += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
    return reinterpret_cast<T*>(p);
  }
};

// A 16-bit matrix as it is stored: rows of cols, pitch ld.
struct Mat {
  const void* p;
  int64_t ld, rows, cols;
  const uint16_t* u16() const { return static_cast<const uint16_t*>(p); }
};

// Direct-to-LDS loads take rows of whole aligned 16-byte chunks; other
// matrices are copied zero-padded first. (The copy of a misaligned weight
// costs its bytes twice more; a program that lays its weights out at such a
// pitch meets it with every call.)
bool loads_direct(const Mat& m) {
  return (reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && m.ld % 8 == 0 && m.cols % 8 == 0 && m.ld < ac::DL_MAX_LD;
}
struct Copies {
  Scratch* s;
  bool all;  // (sizing) as if every matrix were misaligned
  ac::PadArgs args = {};
  Mat operator()(Mat m) {
    if (m.rows == 0 || m.cols == 0 || (!all && loads_direct(m))) return m;
    const int64_t ld = up8(m.cols);
    uint16_t* d = s->take<uint16_t>(m.rows * ld);
    ac::PadMat& p = args.m[args.n++];
    p.src = m.u16();
    p.dst = d;
    p.ld_src = m.ld;
    p.ld_dst = ld;
    p.rows = m.rows;
    p.cols = m.cols;
    m.p = d;
    m.ld = ld;
    return m;
  }
  // two matrices that a kernel reads at one pitch
  void pair(Mat* a, Mat* b) {
    const bool was = all;
    all = all || !loads_direct(*a) || !loads_direct(*b);
    *a = (*this)(*a);
    *b = (*this)(*b);
    all = was;
  }
  // makes them, in one launch
  hipError_t run(hipStream_t st, int* launches) {
    if (args.n == 0) return hipSuccess;
    ++*launches;
    return ac::launch_pad_many(args, st);
  }
};

// How a product (or several of one depth) is tiled and split along K: the
// configuration that the planner's calibrated costs of the direct-to-LDS tiles
// make fastest.
enum FfnKind {
  FFN_GATED = 0,  // weights column by column
  FFN_DGATE = 1,
  FFN_DX = 2,
  FFN_DW = 3,
  FFN_ADAPTER = 4,
  FFN_GATED_ROWS = 5  // and row by row: the tile takes 128 features of each at least
};
struct FfnChoice {
  ac::FfnTile tile = {128, 256, 3};
  bool fused = false;  // the tile's own epilogue (k_gated, k_dgate, k_adapter), else sums of partials
  int pk = 1, kper = 1;
};
constexpr int64_t ADAPTER_BESIDE = 64;  // rows up to which T may be made in the launch of the partial sums
constexpr struct {
  int bm, bn, stages, cfg;  // cfg: direct-to-LDS configuration of the planner
  bool gated, dgate, dw;    // kernels that exist beside k_multi with row-stored A (k_adapter: as k_dgate)
} kFfnTiles[] = {{256, 256, 2, 0, true, true, true},    {128, 256, 3, 2, true, false, true},
                 {128, 128, 2, 9, true, true, true},    {128, 128, 3, 3, true, true, true},
                 {64, 256, 4, 12, false, false, false}, {32, 256, 4, 11, false, false, false},
                 {32, 128, 4, 13, false, false, false}};

// What the planner's costs leave out of these kernels, seconds: fitted to the
// times of all choices of 128 drawn sizes of adapters and of 83 of the block (M
// from 1 to 8192). How much slower than the fastest choice of its size the
// chosen one is, on average: adapters 1.7 %, gated projections 1.7 (columns) or
// 2.3 (rows), dgate 1.9, dX and Y 1.6, weight gradients 1.1; by the planner's
// costs alone, and without the three-stage tile, 8.0, 2.5, 2.5, 4.7, 3.3, 3.4 and
// more.
double unplanned(FfnKind kind, const ac::FfnTile& tile, int64_t M, int64_t N, int64_t K, int pk, bool fused) {
  const double mn = (double)M * (double)N;
  const bool two_a_cu = tile.bn < 256 && tile.stages == 2;
  if (fused) {
    // Epilogues that read and write several matrices: a tile that has its CU to
    // itself does them with nothing beside it, 128 x 128 of two stages, two to a
    // CU, under the other's products. (128 x 256 with these epilogues was the
    // fastest for 2 of 37 sizes, by 3 and 4 %, and is left out; gated it is the
    // only one below 256 x 256 for weights row by row.)
    if (kind == FFN_DGATE) return tile.bn < 256 ? 0 : 3e-12 * mn;
    if (kind == FFN_ADAPTER) return two_a_cu ? 0 : tile.bn < 256 ? 1e-12 * mn : 2e-12 * mn;
    return kind == FFN_GATED_ROWS ? 0 : tile.bn < 256 ? -1.5e-12 * mn : tile.bm < 256 ? 0 : 0.5e-12 * mn;
  }
  // sums of partitions: trips to memory, and each partition's share of them
  // (k_adapter_sum reads T and up besides; gated: N counts both products)
  if (kind == FFN_ADAPTER) {
    double t = 1e-6 * pk + (4e-12 + 1.5e-12 * pk) * mn;
    // Few rows: T in a launch of its own, or beside 32 x 128, whose tiles share
    // CUs with it where they are nearly as many. us by tiles, rank 16: 16 rows of
    // 4096 x 4096 (N x K) 192: 15.1, 224: 15.2, 256: 17.9; of 8192 x 8192 192: 26.8,
    // 256: 33.4; 32 of 2048 x 8192 192: 21.2, 224: 21.7, 256: 24.8. (Tiles of one
    // row of tiles: with both rows of 33 to 64 rows counted twelve choices of 150
    // sizes changed, nine for the worse, 4 % on average.)
    if (M <= ADAPTER_BESIDE && !(tile.bm == 32 && tile.bn == 128)) t += 8e-6;
    if (M <= ADAPTER_BESIDE && tile.bm == 32 && tile.bn == 128 && cdiv(N, 128) * pk > 208) t += 1e-9 * (double)K;
    return t;
  }
  const double each = kind == FFN_GATED || kind == FFN_GATED_ROWS ? 0.375e-12 : 0.75e-12;
  return pk > 1 ? 2e-6 + (0.75e-6 + each * mn) * pk : 0;
}

// Choices made under the planner's profile; cleared with its plans, which no
// call may run beside.
std::mutex g_choices_mu;
std::map<std::tuple<int, int64_t, int64_t, int64_t, int>, FfnChoice> g_choices;

// `blocks`: the product's 64-deep k-blocks; they are not cdiv(K, 64) where K is
// in two segments, each rounded up to blocks of its own.
const FfnChoice& ffn_choice(FfnKind kind, int64_t M, int64_t N, int64_t K, int blocks) {
  const auto key = std::make_tuple((int)kind, M, N, K, blocks);
  std::lock_guard<std::mutex> lk(g_choices_mu);
  auto it = g_choices.find(key);
  if (it != g_choices.end()) return it->second;
  const adaptcore_hw_t hw = ac::op_hw();
  FfnChoice best;  // (of a product of depth 0: a tile that has every epilogue of the kind)
  best.kper = std::max(1, blocks);
  const bool gated = kind == FFN_GATED || kind == FFN_GATED_ROWS;
  const bool sums = gated || kind == FFN_DGATE || kind == FFN_ADAPTER;  // one partition may need them too
  best.fused = sums;
  if (!gated) best.tile = {128, 128, 2};
  double t_best = INFINITY;  // (costs may be negative: a correction is relative to the other tiles)
  const ac::Shape s{M, up8(N), up8(K), AC_BF16_BF16OUT, AC_LAYOUT_ROW_ROW};
  for (const auto& c : kFfnTiles) {
    if (kind == FFN_DW && !c.dw) continue;
    for (int pk : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64}) {
      if (blocks < 1 || pk > blocks) break;
      const int kper = (int)cdiv(blocks, pk);
      if (cdiv(blocks, kper) != pk) continue;
      // (adapters: up to a tile's rows may each have an adapter of its own, which
      // k_adapter takes four at a time within one workgroup, k_adapter_sum over the
      // grid: 79 rows of 49 requests on 304 x 368 29 and 14.5 us)
      const bool fused = pk == 1 && (kind != FFN_ADAPTER || M > 128) && (gated ? c.gated && (c.bn >= 256 || kind == FFN_GATED) : sums && c.dgate);
      ac::Plan p;
      if (!ac::plan_for_key(s, hw, ac::make_variant_key(ac::FAM_DL, c.cfg, 1, pk, s.dtype, 0), &p)) continue;
      double t = p.predicted;
      t += unplanned(kind, {c.bm, c.bn, c.stages}, M, N, K, pk, fused);
      // one partition without an epilogue of its own: its sums kernel
      if (pk == 1 && sums && !fused)
        t += hw.t_launch + 8.0 * (double)M * (double)N / (hw.hbm_bw * hw.hbm_eta);
      if (t < t_best) {
        t_best = t;
        best.tile = {c.bm, c.bn, c.stages};
        best.pk = pk;
        best.kper = kper;
        best.fused = fused;
      }
    }
  }
  return g_choices[key] = best;
}

// A tile as the lists of kernels name it.
std::string name(const ac::FfnTile& t) {
  return "<" + std::to_string(t.bm) + ", " + std::to_string(t.bn) + (t.bm == t.bn && t.stages == 3 ? ", 3>" : ">");
}

// Tile counts and partial buffers of a launch.
adaptcore_status ffn_tiles(ac::MultiArgs* a, const FfnChoice& c, Scratch* s, bool partials) {
  a->pk = c.pk;
  a->kper = c.kper;
  if ((int64_t)c.pk * c.kper < a->blocks) return ac::op_fail(AC_ERR_INTERNAL, "the split leaves k-blocks out");
  int64_t tiles = 0;
  for (int i = 0; i < a->n; ++i) {
    ac::MultiProd& p = a->p[i];
    // (a tile's loads are 32-bit byte offsets from its first row)
    if (a->blocks > 0 && (p.lda > ac::DL_MAX_LD || p.ldb > ac::DL_MAX_LD))
      return ac::op_fail(AC_ERR_INTERNAL, "operand pitch past the tile's offsets");
    const int64_t tm = cdiv(p.M, c.tile.bm), tn = cdiv(p.N, c.tile.bn);
    tiles += tm * tn;
    if (tm >= (1 << 30) || tn >= (1 << 30) || tiles >= (1LL << 31) / 256) return unsupported("launch grid too large");
    p.tiles_m = (int)tm;
    p.tiles_n = (int)tn;
    p.ldp = up8(p.N);
    p.part = partials ? s->take<float>((int64_t)c.pk * p.M * p.ldp) : nullptr;
  }
  return AC_OK;
}

// C (M x N) = A B with A as rows of K (or, a_rows, stored as K rows of M) and
// B as K rows of N (or, b_cols, N rows of K).
ac::MultiProd product(int64_t M, int64_t N, int64_t K, const Mat& A, bool a_rows, const Mat& B, bool b_cols, void* C,
                      int64_t ldc) {
  ac::MultiProd p;
  std::memset(&p, 0, sizeof p);
  p.A = A.u16();
  p.B = B.u16();
  p.lda = A.ld;
  p.ldb = B.ld;
  p.M = M;
  p.N = N;
  p.eA = a_rows ? up8(M) : M;
  p.eB = b_cols ? N : up8(N);
  p.kA = a_rows ? K : up8(K);
  p.kB = b_cols ? up8(K) : K;
  p.C = C;
  p.ldc = ldc;
  return p;
}

struct FfnSize {
  int64_t M, D, F;
  int32_t type;
  uint32_t layouts;
  int32_t act;
  bool up_col() const { return (layouts & AC_FFN_UP_COL) != 0; }
  bool down_col() const { return (layouts & AC_FFN_DOWN_COL) != 0; }
  bool f16() const { return type == AC_TYPE_F16; }
  Mat up(const void* p, int64_t ld) const { return up_col() ? Mat{p, ld, F, D} : Mat{p, ld, D, F}; }
  Mat down(const void* p, int64_t ld) const { return down_col() ? Mat{p, ld, D, F} : Mat{p, ld, F, D}; }
};

adaptcore_status ffn_check(const FfnSize& z, uint32_t known_layouts) {
  if (z.M < 0 || z.M >= (1LL << 31) || z.D < 0 || z.D >= (1LL << 22) || z.F < 0 || z.F >= (1LL << 22))
    return invalid("M must be in [0, 2^31), D and F in [0, 2^22)");
  if (z.type != AC_TYPE_BF16 && z.type != AC_TYPE_F16) return unsupported("the block's type must be bf16 or fp16");
  if (z.layouts & ~known_layouts) return unsupported("unknown layout bits");
  if (z.act != AC_ACT_SILU && z.act != AC_ACT_GELU && z.act != AC_ACT_GELU_TANH)
    return unsupported("unknown activation");
  return AC_OK;
}
// A matrix argument of rows x cols elements of `bytes` each.
adaptcore_status mat_check(const void* p, int64_t ld, int64_t rows, int64_t cols, int bytes) {
  if (ld < std::max<int64_t>(1, cols)) return invalid("row pitch smaller than the stored row");
  if (ld >= AC_MAX_LD) return invalid("row pitch must be below 2^23 elements");
  if (rows > 0 && cols > 0 && !p) return invalid("null matrix pointer");
  if (misaligned(p, bytes)) return invalid("pointer not aligned to its element size");
  return AC_OK;
}
adaptcore_status first_bad(std::initializer_list<adaptcore_status> all) {
  for (adaptcore_status s : all)
    if (s != AC_OK) return s;
  return AC_OK;
}

// Whether `nb` products of M rows, N columns and depth K run on k_rows: few
// rows, weights stored column by column, and faster than the split tiles with
// their sums. us: 2 + what is longer of all weights at 4.2 TB/s and the
// workgroups of one of 256 CUs at 34 GB/s, which read A's rows too, against 9 + all
// weights at 6.5 TB/s. Fitted to the times of both for 500 drawn sizes of 1 to 32
// rows, weights from memory; of 250 others the chosen one is 0.5 % slower than
// the faster on average, at worst 1.45 times. In a graph, us, with 16 and with 32
// rows:
//                       512 x 1536     4096 x 4096    2048 x 8192    8192 x 2048    4096 x 14336
//   both projections
//     k_rows             3.8   4.6     16.9   19.8    17.4   20.4    25.6   31.6    54.6   64.9
//     split and sums     6.7   6.9     18.8   20.0    18.7   19.1    20.7   21.1    48.2   52.4
//   Y, of the transposed size
//     k_rows             4.8   6.4      9.9   13.0    16.7   23.0     9.8   14.1    28.5   40.6
//     its own plan       6.4   6.8     11.5   12.6    12.2   12.9    11.8   12.4    24.1   25.1
// Weights that the tiles would copy first stay here.
bool rows_kernel(int64_t M, int64_t N, int64_t K, int nb, bool col, bool direct) {
  if (!col || K < 1 || M > ac::FFN_ROWS_MAX) return false;
  if (!direct) return true;
  const double bytes = 2.0 * nb * (double)N * (double)K, groups = std::ceil((double)cdiv(N, 16) / 256.0);
  const double cu = 2.0 * (double)K * (16.0 * nb + (M <= 16 ? 16.0 : 32.0)) * groups;
  return 2.0 + std::max(bytes / 4.2e6, cu / 34e3) <= 9.0 + bytes / 6.5e6;
}

// Misaligned projections of few rows: both products in fp32 on their own plans,
// written and read once more (16 M F bytes), unless zero-padded copies move
// less.
bool plain_projections(const FfnSize& z, bool direct) {
  return !direct && z.D > 0 && 16 * z.M * z.F <= 4 * (2 * z.D * z.F + z.M * z.D);
}

#define FFN_CALL(z, fn, ...) ((z).f16() ? ac::f16::fn(__VA_ARGS__) : ac::fn(__VA_ARGS__))

struct FfnForward {
  Mat x, wg, wu, wd, h, y;  // wd and y: unused where `down` is false
  void *g, *u;
  int64_t ldg;
  bool down;  // the whole block
};

// The block, or its first half. Counts the workspace, or (s->base) launches.
// `all`: as if every operand were misaligned.
adaptcore_status run_ffn(const FfnSize& z, FfnForward f, Scratch* s, hipStream_t st, bool all, int* launches) {
  const bool run = s->base != nullptr;
  const int32_t dt16 = z.f16() ? AC_F16_F16OUT : AC_BF16_BF16OUT, dt32 = z.f16() ? AC_F16_F32OUT : AC_BF16_F32OUT;
  const uint32_t up_lay = z.up_col() ? AC_LAYOUT_B_COL : 0, down_lay = z.down_col() ? AC_LAYOUT_B_COL : 0;
  const bool up_direct = !all && loads_direct(f.x) && loads_direct(f.wg) && loads_direct(f.wu);
  const bool down_direct = !all && loads_direct(f.h) && loads_direct(f.wd);
  const bool gated = z.M > 0 && z.F > 0;
  const bool up_rows = rows_kernel(z.M, z.F, z.D, 2, z.up_col(), up_direct);
  const bool up_plain = !up_rows && plain_projections(z, up_direct);
  const bool down_rows = rows_kernel(z.M, z.D, z.F, 1, z.down_col(), down_direct);
  // Y = H Wd: as dX on tiles, the operands of odd sizes padded by the first
  // half, which writes H once more. Few rows: on the product's own plan.
  const bool down_tiles = f.down && !down_rows && z.F > 0 && z.D > 0 && z.M > 64 &&
                          (down_direct || (!up_rows && !up_plain));
  Copies copy = {s, all};
  if (gated && !up_rows && !up_plain) {
    f.x = copy(f.x);
    copy.pair(&f.wg, &f.wu);
  }
  Mat h2 = f.h;
  if (down_tiles && gated) {
    f.wd = copy(f.wd);
    if (all || !loads_direct(f.h)) {
      h2.ld = up8(z.F);
      h2.p = s->take<uint16_t>(z.M * h2.ld);
    }
  }
  const bool second_h = h2.ld != f.h.ld || h2.p != f.h.p;
  hipError_t e = hipSuccess;
  int n = 0;
  if (run) e = copy.run(st, &n);

  if (gated && up_rows) {
    const ac::RowsArgs r = {f.x.u16(), f.wg.u16(), f.wu.u16(), f.x.ld, f.wg.ld, z.M, z.F, z.D, const_cast<void*>(f.h.p),
                            f.h.ld, static_cast<uint16_t*>(f.g), static_cast<uint16_t*>(f.u), f.ldg, z.act};
    if (run && e == hipSuccess) e = FFN_CALL(z, ffn_rows, r, true, st);
    ++n;
  } else if (gated) {
    const int blocks = (int)cdiv(z.D, 64);
    const FfnChoice c = up_plain ? FfnChoice() : ffn_choice(z.up_col() ? FFN_GATED : FFN_GATED_ROWS, z.M, 2 * z.F, z.D, blocks);
    const bool fused = c.fused && !up_plain;
    ac::MultiArgs a;
    std::memset(&a, 0, sizeof a);
    a.n = 2;
    a.blocks = a.seg = up_plain ? 0 : blocks;  // (plain: none of its products are launched, its sums are)
    a.p[0] = product(z.M, z.F, z.D, f.x, false, f.wg, z.up_col(), nullptr, 0);
    a.p[1] = product(z.M, z.F, z.D, f.x, false, f.wu, z.up_col(), nullptr, 0);
    FfnChoice half = c;
    if (fused) half.tile.bn /= 2;  // a tile's columns are two of each feature
    if (const adaptcore_status rc = ffn_tiles(&a, half, s, !fused)) return rc;
    ac::GatedArgs g;
    std::memset(&g, 0, sizeof g);
    g.X = f.x.u16();
    g.Wg = f.wg.u16();
    g.Wu = f.wu.u16();
    g.ldx = f.x.ld;
    g.ldw = f.wg.ld;
    g.M = z.M;
    g.F = z.F;
    g.eF = a.p[0].eB;
    g.kX = a.p[0].kA;
    g.kW = a.p[0].kB;
    g.H = static_cast<uint16_t*>(const_cast<void*>(f.h.p));
    g.ldh = f.h.ld;
    g.H2 = second_h ? static_cast<uint16_t*>(const_cast<void*>(h2.p)) : nullptr;
    g.ldh2 = h2.ld;
    g.G = static_cast<uint16_t*>(f.g);
    g.U = static_cast<uint16_t*>(f.u);
    g.ldg = f.ldg;
    g.act = z.act;
    if (up_plain) {
      const int64_t bytes = ac::op_matmul_workspace(z.M, z.F, z.D, dt32, up_lay);
      char* ws = s->take<char>(std::max<int64_t>(bytes, 1));
      for (int i = 0; i < 2 && run && e == hipSuccess; ++i) {
        const Mat& w = i ? f.wu : f.wg;
        const adaptcore_status rc = ac::op_matmul(z.M, z.F, z.D, dt32, up_lay, f.x.p, f.x.ld, w.p, w.ld, a.p[i].part,
                                                  a.p[i].ldp, st, ws, bytes);
        if (rc != AC_OK) return rc;
      }
      if (run && e == hipSuccess) e = FFN_CALL(z, ffn_gated_sum, a, g, st);
      ++n;
    } else if (fused) {
      g.tiles_m = a.p[0].tiles_m;
      g.tiles_n = a.p[0].tiles_n;
      if (run && e == hipSuccess) e = FFN_CALL(z, ffn_gated, c.tile, g, (int)up_lay, st);
      ++n;
    } else {
      if (run && e == hipSuccess) e = FFN_CALL(z, ffn_multi, c.tile, a, (int)up_lay, 2, st);
      if (run && e == hipSuccess) e = FFN_CALL(z, ffn_gated_sum, a, g, st);
      n += 2;
    }
  }

  if (f.down && z.M > 0 && z.D > 0) {
    if (down_rows) {
      ac::RowsArgs r;
      std::memset(&r, 0, sizeof r);
      r.A = f.h.u16();
      r.B = f.wd.u16();
      r.lda = f.h.ld;
      r.ldb = f.wd.ld;
      r.M = z.M;
      r.N = z.D;
      r.K = z.F;
      r.C = const_cast<void*>(f.y.p);
      r.ldc = f.y.ld;
      if (run && e == hipSuccess) e = FFN_CALL(z, ffn_rows, r, false, st);
      ++n;
    } else if (down_tiles) {
      ac::MultiArgs a;
      std::memset(&a, 0, sizeof a);
      a.n = 1;
      a.blocks = a.seg = (int)cdiv(z.F, 64);
      a.p[0] = product(z.M, z.D, z.F, h2, false, f.wd, z.down_col(), const_cast<void*>(f.y.p), f.y.ld);
      const FfnChoice& c = ffn_choice(FFN_DX, z.M, z.D, z.F, a.blocks);
      if (const adaptcore_status rc = ffn_tiles(&a, c, s, c.pk > 1)) return rc;
      if (run && e == hipSuccess) e = FFN_CALL(z, ffn_multi, c.tile, a, (int)down_lay, 1, st);
      if (run && e == hipSuccess && c.pk > 1) e = FFN_CALL(z, ffn_plain_sum, a, 1, st);
      n += c.pk > 1 ? 2 : 1;
    } else {
      const int64_t bytes = ac::op_matmul_workspace(z.M, z.D, z.F, dt16, down_lay);
      char* ws = s->take<char>(std::max<int64_t>(bytes, 1));
      if (run && e == hipSuccess) {
        const adaptcore_status rc = ac::op_matmul(z.M, z.D, z.F, dt16, down_lay, f.h.p, f.h.ld, f.wd.p, f.wd.ld,
                                                  const_cast<void*>(f.y.p), f.y.ld, st, ws, bytes);
        if (rc != AC_OK) return rc;
      }
    }
  }
  *launches += n;
  return launched(e, 0);
}

struct FfnBackward {
  Mat dy, x, wg, wu, wd, g, u, h;
  void* dx;
  int64_t lddx;
  int32_t grad_type;
  void *dwg, *dwu, *dwd;
  int64_t lddw, lddd;
};

adaptcore_status run_ffn_backward(const FfnSize& z, FfnBackward b, Scratch* s, hipStream_t st, bool all,
                                  int* launches) {
  const bool run = s->base != nullptr;
  if (z.D == 0) return AC_OK;  // no element of dX or of a weight
  const bool want_up = b.dwg != nullptr, want_down = b.dwd != nullptr, want_x = b.dx != nullptr && z.M > 0;
  const int64_t F8 = up8(z.F);
  const bool gates = (want_up || want_x) && z.M > 0 && z.F > 0;
  Copies copy = {s, all};
  b.dy = copy(b.dy);
  if (want_up) b.x = copy(b.x);
  if (want_down) b.h = copy(b.h);
  if (gates) b.wd = copy(b.wd);
  if (want_x) copy.pair(&b.wg, &b.wu);
  int n = 0;
  hipError_t e = hipSuccess;
  if (run) e = copy.run(st, &n);
  // dG and dU, each of the pitch the tile's loads take (side by side they would
  // be twice as far from row to row)
  Mat dg = {nullptr, F8, z.M, z.F}, du = dg;
  if (gates) {
    uint16_t* const pg = s->take<uint16_t>(z.M * F8);
    uint16_t* const pu = s->take<uint16_t>(z.M * F8);
    dg.p = pg;
    du.p = pu;
    const int blocks = (int)cdiv(z.D, 64);
    const FfnChoice& c = ffn_choice(FFN_DGATE, z.M, z.F, z.D, blocks);
    const int lay = z.down_col() ? 0 : AC_LAYOUT_B_COL;  // B = Wd^T
    ac::MultiArgs a;
    std::memset(&a, 0, sizeof a);
    a.n = 1;
    a.blocks = a.seg = blocks;
    a.p[0] = product(z.M, z.F, z.D, b.dy, false, b.wd, !z.down_col(), nullptr, 0);
    if (const adaptcore_status rc = ffn_tiles(&a, c, s, !c.fused)) return rc;
    const ac::DgateArgs d = {b.g.u16(), b.u.u16(), b.g.ld, pg, pu, F8, z.act};
    if (run && e == hipSuccess) {
      if (c.fused) {
        e = FFN_CALL(z, ffn_dgate, c.tile, a, d, lay, st);
        n += 1;
      } else {
        e = FFN_CALL(z, ffn_multi, c.tile, a, lay, 2, st);
        if (e == hipSuccess) e = FFN_CALL(z, ffn_dgate_sum, a, d, st);
        n += 2;
      }
    }
  }
  if (want_x) {
    const int seg = (int)cdiv(z.F, 64);
    const FfnChoice& c = ffn_choice(FFN_DX, z.M, z.D, 2 * z.F, 2 * seg);
    const int lay = z.up_col() ? 0 : AC_LAYOUT_B_COL;  // B = Wg^T, Wu^T
    ac::MultiArgs a;
    std::memset(&a, 0, sizeof a);
    a.n = 1;
    a.blocks = 2 * seg;
    a.seg = seg;
    a.p[0] = product(z.M, z.D, z.F, dg, false, b.wg, !z.up_col(), b.dx, b.lddx);
    a.p[0].A2 = du.u16();
    a.p[0].B2 = b.wu.u16();
    if (const adaptcore_status rc = ffn_tiles(&a, c, s, c.pk > 1)) return rc;
    if (run && e == hipSuccess) {
      e = FFN_CALL(z, ffn_multi, c.tile, a, lay, 1, st);
      if (e == hipSuccess && c.pk > 1) e = FFN_CALL(z, ffn_plain_sum, a, 1, st);
      n += c.pk > 1 ? 2 : 1;
    }
  }
  if ((want_up || want_down) && z.F > 0) {
    ac::MultiArgs a;
    std::memset(&a, 0, sizeof a);
    a.blocks = a.seg = (int)cdiv(z.M, 64);
    // (the left operand's and the right one's rows are both the tokens)
    if (want_up) {
      for (int i = 0; i < 2; ++i) {
        const Mat& d = i ? du : dg;
        void* out = i ? b.dwu : b.dwg;
        a.p[a.n++] = z.up_col() ? product(z.F, z.D, z.M, d, true, b.x, false, out, b.lddw)
                                : product(z.D, z.F, z.M, b.x, true, d, false, out, b.lddw);
      }
    }
    if (want_down)
      a.p[a.n++] = z.down_col() ? product(z.D, z.F, z.M, b.dy, true, b.h, false, b.dwd, b.lddd)
                                : product(z.F, z.D, z.M, b.h, true, b.dy, false, b.dwd, b.lddd);
    const FfnChoice& c = ffn_choice(FFN_DW, a.n * z.F, z.D, z.M, a.blocks);
    if (const adaptcore_status rc = ffn_tiles(&a, c, s, c.pk > 1)) return rc;
    const int out = b.grad_type == AC_TYPE_F32 ? 0 : 1;
    if (run && e == hipSuccess) {
      e = FFN_CALL(z, ffn_multi, c.tile, a, AC_LAYOUT_A_COL, out, st);
      if (e == hipSuccess && c.pk > 1) e = FFN_CALL(z, ffn_plain_sum, a, out, st);
      n += c.pk > 1 ? 2 : 1;
    }
  }
  *launches += n;
  return launched(e, 0);
}

// ---- adapters beside a shared projection
struct AdapterCall {
  int64_t M, N, K;
  int32_t dtype;
  bool w_col;
  Mat x, w;
  ac::AdapterArgs g;  // everything but T
};

// How a call runs: R its rank (0: no adapters), direct: X and W as they lie.
struct AdapterWay {
  const FfnChoice* how;
  bool plain;   // the shared product in fp32 on its own plan
  bool fused;   // k_adapter, else k_adapter_sum
  bool beside;  // T in the launch of the partial sums
};
AdapterWay adapter_way(int64_t M, int64_t N, int64_t K, int64_t R, bool direct) {
  AdapterWay w;
  w.how = &ffn_choice(FFN_ADAPTER, M, N, K, (int)cdiv(K, 64));
  // Misaligned operands: the product's own plan reads them as they are, or
  // copies; its fp32 result is written and read once more (8 M N bytes), unless
  // zero-padded copies of both for the tile move less.
  w.plain = !direct && 2 * M * N <= K * (M + N);
  w.fused = w.how->fused && !w.plain;
  // few rows of few adapters: the tile leaves room for a second workgroup on
  // every CU
  w.beside = R > 0 && R <= 64 && !w.fused && !w.plain && w.how->tile.bm == 32 && w.how->tile.bn == 128 &&
             M <= ADAPTER_BESIDE;
  return w;
}

adaptcore_status run_adapter(const AdapterCall& c, Scratch* s, hipStream_t st, bool all, int* launches) {
  if (c.M == 0 || c.N == 0) return AC_OK;
  const bool f16 = ac::dtype_f16_input(c.dtype), out16 = ac::dtype_out16(c.dtype);
  ac::AdapterArgs g = c.g;
  const bool low_rank = g.n > 0 && g.R > 0;
  if (!low_rank) g.n = 0;
  g.ldt = cdiv(g.R, 16) * 16;
  const bool direct = !all && loads_direct(c.x) && loads_direct(c.w);
  const int blocks = (int)cdiv(c.K, 64);
  const AdapterWay way = adapter_way(c.M, c.N, c.K, low_rank ? g.R : 0, direct);
  const FfnChoice& how = *way.how;
  const bool plain = way.plain, fused = way.fused, beside = way.beside;
  g.T = low_rank ? s->take<char>(c.M * g.ldt * (fused ? 2 : 4)) : nullptr;
  ac::MultiArgs a;
  std::memset(&a, 0, sizeof a);
  a.n = 1;
  a.blocks = a.seg = blocks;
  char* mm_ws = nullptr;
  int64_t mm_bytes = 0;
  Copies copy = {s, all};
  const int32_t f32 = f16 ? AC_F16_F32OUT : AC_BF16_F32OUT;
  const uint32_t lay = c.w_col ? AC_LAYOUT_B_COL : 0;
  if (plain) {
    a.pk = a.kper = 1;
    a.p[0].M = c.M;
    a.p[0].N = c.N;
    a.p[0].ldp = up8(c.N);
    a.p[0].part = s->take<float>(c.M * a.p[0].ldp);
    mm_bytes = ac::op_matmul_workspace(c.M, c.N, c.K, f32, lay);
    mm_ws = s->take<char>(std::max<int64_t>(mm_bytes, 1));
  } else {
    a.p[0] = product(c.M, c.N, c.K, copy(c.x), false, copy(c.w), c.w_col, nullptr, 0);
    if (const adaptcore_status rc = ffn_tiles(&a, how, s, !fused)) return rc;
  }
  if (!s->base) return AC_OK;
  int n = 0;
  hipError_t e = copy.run(st, &n);
  if (e == hipSuccess && low_rank && !beside) {
    e = f16 ? ac::f16::adapter_shrink(g, fused, st) : ac::adapter_shrink(g, fused, st);
    ++n;
  }
  if (e == hipSuccess && fused) {
    e = f16 ? ac::f16::adapter_tile(how.tile, a, g, (int)lay, out16, st)
            : ac::adapter_tile(how.tile, a, g, (int)lay, out16, st);
    ++n;
  } else if (e == hipSuccess) {
    if (plain) {
      const adaptcore_status rc = ac::op_matmul(c.M, c.N, c.K, f32, lay, c.x.p, c.x.ld, c.w.p, c.w.ld, a.p[0].part,
                                                a.p[0].ldp, st, mm_ws, mm_bytes);
      if (rc != AC_OK) return rc;
    } else if (beside) {
      e = f16 ? ac::f16::adapter_multi_shrink(a, g, (int)lay, st) : ac::adapter_multi_shrink(a, g, (int)lay, st);
      ++n;
    } else {
      e = f16 ? ac::f16::ffn_multi(how.tile, a, (int)lay, 2, st) : ac::ffn_multi(how.tile, a, (int)lay, 2, st);
      ++n;
    }
    if (e == hipSuccess) e = f16 ? ac::f16::adapter_sum(a, g, out16, st) : ac::adapter_sum(a, g, out16, st);
    ++n;
  }
  *launches += n;
  return launched(e, 0);
}

adaptcore_status adapter_size(int64_t M, int64_t N, int64_t K, int32_t dtype, uint32_t layouts, int64_t n, int64_t R) {
  if (M < 0 || M >= (1LL << 22) || N < 0 || N >= (1LL << 22) || K < 0 || K >= (1LL << 22))
    return invalid("M, N and K must be in [0, 2^22)");
  if (n < 0 || n >= (1LL << 31) || R < 0 || R > 4096) return invalid("adapters must be in [0, 2^31), rank in [0, 4096]");
  if (dtype < AC_BF16_F32OUT || dtype > AC_F16_F16OUT) return unsupported("unknown dtype");
  if (layouts & ~(uint32_t)AC_LAYOUT_B_COL) return unsupported("X is row-major, W row-major or column-major");
  return AC_OK;
}

// Runs f twice: counting the workspace, then on it.
template <class F>
adaptcore_status with_scratch(hipStream_t st, F f) {
  Scratch s;
  int n = 0;
  adaptcore_status rc = f(&s, &n);
  if (rc != AC_OK) return rc;
  char none[1];
  s.base = none;  // (no workspace needed: any address, nothing is taken from it)
  std::unique_lock<std::mutex> hold;
  if (s.used > 0) rc = ac::op_workspace(st, s.used, &s.base, &hold);
  if (rc != AC_OK) return rc;
  s.used = 0;
  n = 0;
  rc = f(&s, &n);
  if (rc == AC_OK) ac::op_count_launches(n);
  return rc;
}

adaptcore_status gated_args(const FfnSize& z, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw,
                            void* H, int64_t ldh, void* G, void* U, int64_t ldg) {
  if ((G == nullptr) != (U == nullptr)) return invalid("G and U must both be given or both be null");
  const Mat g = z.up(Wg, ldw);
  return first_bad({mat_check(X, ldx, z.M, z.D, 2), mat_check(Wg, ldw, g.rows, g.cols, 2),
                    mat_check(Wu, ldw, g.rows, g.cols, 2), mat_check(H, ldh, z.M, z.F, 2),
                    G ? mat_check(G, ldg, z.M, z.F, 2) : AC_OK, G ? mat_check(U, ldg, z.M, z.F, 2) : AC_OK});
}

}  // namespace

namespace ac {
void op_clear_choices() {
  std::lock_guard<std::mutex> lk(g_choices_mu);
  g_choices.clear();
}
}  // namespace ac

extern "C" {

adaptcore_status adaptcore_gated_matmul(int64_t M, int64_t D, int64_t F, int32_t type, uint32_t layouts,
                                        int32_t activation, const void* X, int64_t ldx, const void* Wg, const void* Wu,
                                        int64_t ldw, void* H, int64_t ldh, void* G, void* U, int64_t ldg,
                                        void* stream) {
  return guarded([&] {
    const FfnSize z = {M, D, F, type, layouts, activation};
    adaptcore_status st = ffn_check(z, AC_FFN_UP_COL);
    if (st == AC_OK) st = gated_args(z, X, ldx, Wg, Wu, ldw, H, ldh, G, U, ldg);
    if (st != AC_OK || M == 0 || F == 0) return st;
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return with_scratch(s, [&](Scratch* w, int* n) {
      return run_ffn(z, {{X, ldx, M, D}, z.up(Wg, ldw), z.up(Wu, ldw), {}, {H, ldh, M, F}, {}, G, U, ldg, false}, w, s,
                     false, n);
    });
  });
}

adaptcore_status adaptcore_gated_ffn(int64_t M, int64_t D, int64_t F, int32_t type, uint32_t layouts,
                                     int32_t activation, const void* X, int64_t ldx, const void* Wg, const void* Wu,
                                     int64_t ldw, const void* Wd, int64_t ldd, void* H, int64_t ldh, void* G, void* U,
                                     int64_t ldg, void* Y, int64_t ldy, void* stream) {
  return guarded([&] {
    const FfnSize z = {M, D, F, type, layouts, activation};
    adaptcore_status st = ffn_check(z, AC_FFN_UP_COL | AC_FFN_DOWN_COL);
    if (st == AC_OK) st = gated_args(z, X, ldx, Wg, Wu, ldw, H, ldh, G, U, ldg);
    const Mat wd = z.down(Wd, ldd);
    if (st == AC_OK) st = first_bad({mat_check(Wd, ldd, wd.rows, wd.cols, 2), mat_check(Y, ldy, M, D, 2)});
    if (st != AC_OK || M == 0) return st;
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return with_scratch(s, [&](Scratch* w, int* n) {
      return run_ffn(z, {{X, ldx, M, D}, z.up(Wg, ldw), z.up(Wu, ldw), wd, {H, ldh, M, F}, {Y, ldy, M, D}, G, U, ldg,
                         true}, w, s, false, n);
    });
  });
}

adaptcore_status adaptcore_gated_ffn_backward(int64_t M, int64_t D, int64_t F, int32_t type, uint32_t layouts,
                                              int32_t activation, const void* dY, int64_t lddy, const void* X,
                                              int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, const void* Wd,
                                              int64_t ldd, const void* G, const void* U, int64_t ldg, const void* H,
                                              int64_t ldh, void* dX, int64_t lddx, int32_t grad_type, void* dWg,
                                              void* dWu, int64_t lddw, void* dWd, int64_t lddd, void* stream) {
  return guarded([&] {
    const FfnSize z = {M, D, F, type, layouts, activation};
    adaptcore_status st = ffn_check(z, AC_FFN_UP_COL | AC_FFN_DOWN_COL);
    if (st != AC_OK) return st;
    if (grad_type != AC_TYPE_F32 && grad_type != type)
      return unsupported("the weight gradients must be fp32 or of the block's type");
    if ((dWg == nullptr) != (dWu == nullptr)) return invalid("dWg and dWu must both be given or both be null");
    const Mat up = z.up(nullptr, 0), down = z.down(nullptr, 0);
    const int gb = type_bytes(grad_type);
    st = first_bad({mat_check(dY, lddy, M, D, 2), mat_check(X, ldx, M, D, 2), mat_check(Wg, ldw, up.rows, up.cols, 2),
                    mat_check(Wu, ldw, up.rows, up.cols, 2), mat_check(Wd, ldd, down.rows, down.cols, 2),
                    mat_check(G, ldg, M, F, 2), mat_check(U, ldg, M, F, 2), mat_check(H, ldh, M, F, 2),
                    dX ? mat_check(dX, lddx, M, D, 2) : AC_OK, dWg ? mat_check(dWg, lddw, up.rows, up.cols, gb) : AC_OK,
                    dWg ? mat_check(dWu, lddw, up.rows, up.cols, gb) : AC_OK,
                    dWd ? mat_check(dWd, lddd, down.rows, down.cols, gb) : AC_OK});
    if (st != AC_OK || D == 0 || (!dX && !dWg && !dWd)) return st;
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const FfnBackward b = {{dY, lddy, M, D}, {X, ldx, M, D}, z.up(Wg, ldw), z.up(Wu, ldw), z.down(Wd, ldd),
                           {G, ldg, M, F},   {U, ldg, M, F}, {H, ldh, M, F}, dX, lddx, grad_type, dWg, dWu, dWd,
                           lddw, lddd};
    return with_scratch(
        s, [&](Scratch* w, int* n) { return run_ffn_backward(z, b, w, s, false, n); });
  });
}

int64_t adaptcore_gated_ffn_workspace(int64_t M, int64_t D, int64_t F, int32_t backward) {
  int64_t bytes = 0;
  const adaptcore_status st = guarded([&] {
    for (uint32_t lay = 0; lay < 4; ++lay) {
      const FfnSize z = {M, D, F, AC_TYPE_BF16, lay, AC_ACT_SILU};
      adaptcore_status rc = ffn_check(z, AC_FFN_UP_COL | AC_FFN_DOWN_COL);
      if (rc != AC_OK) return rc;
      Scratch s;
      int n = 0;
      if (backward) {
        int any = 0;
        for (int wanted = 1; wanted < 4; ++wanted) {  // (fewer products of one launch may be split further)
          void *up = (wanted & 1) ? &any : nullptr, *down = (wanted & 2) ? &any : nullptr;
          const FfnBackward b = {{nullptr, D, M, D}, {nullptr, D, M, D},  z.up(nullptr, 1),   z.up(nullptr, 1),
                                 z.down(nullptr, 1), {nullptr, F, M, F},  {nullptr, F, M, F}, {nullptr, F, M, F},
                                 &any, D, AC_TYPE_F32, up, up, down, F, F};
          s.used = 0;
          rc = run_ffn_backward(z, b, &s, nullptr, true, &n);
          if (rc != AC_OK) return rc;
          bytes = std::max(bytes, s.used);
        }
      } else {
        // every operand misaligned, none, or those of one half
        for (int odd = 0; odd < 4; ++odd) {
          auto mat = [](Mat m, bool bad) {
            m.p = bad ? reinterpret_cast<const void*>(2) : nullptr;
            m.ld = up8(m.cols);
            m.cols = bad ? m.cols : up8(m.cols);
            return m;
          };
          const bool up = (odd & 1) != 0, down = (odd & 2) != 0;
          const FfnForward f = {mat({nullptr, 1, M, D}, up), mat(z.up(nullptr, 1), up), mat(z.up(nullptr, 1), up),
                                mat(z.down(nullptr, 1), down), mat({nullptr, 1, M, F}, down), {nullptr, D, M, D},
                                nullptr, nullptr, 1, true};
          s.used = 0;
          rc = run_ffn(z, f, &s, nullptr, false, &n);
          if (rc != AC_OK) return rc;
          bytes = std::max(bytes, s.used);
        }
        s.used = 0;
      }
      if (rc != AC_OK) return rc;
      bytes = std::max(bytes, s.used);
    }
    return AC_OK;
  });
  return st == AC_OK ? bytes : (int64_t)st;
}

adaptcore_status adaptcore_adapter_matmul(int64_t M, int64_t N, int64_t K, int32_t dtype, uint32_t layouts,
                                          const void* X, int64_t ldx, const void* W, int64_t ldw, int64_t adapters,
                                          int64_t rank, const void* down, int64_t ld_down, int64_t stride_down,
                                          const void* up, int64_t ld_up, int64_t stride_up, const int32_t* index,
                                          const float* scale, const float* bias, void* Y, int64_t ldy, void* stream) {
  return guarded([&] {
    adaptcore_status st = adapter_size(M, N, K, dtype, layouts, adapters, rank);
    if (st != AC_OK) return st;
    const bool col = (layouts & AC_LAYOUT_B_COL) != 0;
    const Mat w = col ? Mat{W, ldw, N, K} : Mat{W, ldw, K, N};
    const bool some = adapters > 0 && rank > 0;
    st = first_bad({mat_check(X, ldx, M, K, 2), mat_check(W, ldw, w.rows, w.cols, 2),
                    mat_check(Y, ldy, M, N, ac::dtype_out_bytes(dtype)),
                    some ? mat_check(down, ld_down, rank, K, 2) : AC_OK, some ? mat_check(up, ld_up, N, rank, 2) : AC_OK});
    if (st != AC_OK) return st;
    const int64_t lim = 1LL << 40;
    if (stride_down < 0 || stride_down >= lim || stride_up < 0 || stride_up >= lim)
      return invalid("the adapters' strides must be in [0, 2^40)");
    if (misaligned(index, 4) || misaligned(scale, 4) || misaligned(bias, 4))
      return invalid("pointer not aligned to its element size");
    if (M == 0 || N == 0) return AC_OK;
    if (some && !index) return invalid("null index pointer");
    st = ac::op_ready();
    if (st != AC_OK) return st;
    AdapterCall c = {M, N, K, dtype, col, {X, ldx, M, K}, w, {}};
    c.g.X = static_cast<const uint16_t*>(X);
    c.g.ldx = ldx;
    c.g.M = M;
    c.g.N = N;
    c.g.K = K;
    c.g.n = (int)adapters;
    c.g.R = (int)rank;
    c.g.down = static_cast<const uint16_t*>(down);
    c.g.ld_down = ld_down;
    c.g.stride_down = stride_down;
    c.g.up = static_cast<const uint16_t*>(up);
    c.g.ld_up = ld_up;
    c.g.stride_up = stride_up;
    c.g.index = index;
    c.g.scale = scale;
    c.g.bias = bias;
    c.g.Y = Y;
    c.g.ldy = ldy;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return with_scratch(s, [&](Scratch* ws, int* n) { return run_adapter(c, ws, s, false, n); });
  });
}

int64_t adaptcore_adapter_workspace(int64_t M, int64_t N, int64_t K, int64_t rank) {
  int64_t bytes = 0;
  const adaptcore_status st = guarded([&] {
    for (int32_t dt : {AC_BF16_F32OUT, AC_F16_F32OUT})
      for (bool col : {false, true})
        for (bool all : {false, true}) {
          const adaptcore_status rc = adapter_size(M, N, K, dt, 0, 1, rank);
          if (rc != AC_OK) return rc;
          AdapterCall c;
          std::memset(&c, 0, sizeof c);
          c.M = M;
          c.N = N;
          c.K = K;
          c.dtype = dt;
          c.w_col = col;
          c.x = {nullptr, up8(K), M, up8(K)};  // (all == false: aligned)
          c.w = col ? Mat{nullptr, up8(K), N, up8(K)} : Mat{nullptr, up8(N), K, up8(N)};
          c.g.n = 1;
          c.g.R = (int)rank;
          Scratch s;
          int n = 0;
          const adaptcore_status r2 = run_adapter(c, &s, nullptr, all, &n);
          if (r2 != AC_OK) return r2;
          bytes = std::max(bytes, s.used);
        }
    return AC_OK;
  });
  return st == AC_OK ? bytes : (int64_t)st;
}

adaptcore_status adaptcore_adapter_kernels(int64_t M, int64_t N, int64_t K, char* buf, int64_t len) {
  return adaptcore_adapter_call_kernels(M, N, K, 1, 4096, buf, len);
}

adaptcore_status adaptcore_adapter_call_kernels(int64_t M, int64_t N, int64_t K, int64_t adapters, int64_t rank,
                                                char* buf, int64_t len) {
  return guarded([&] {
    if (!buf || len < 1) return invalid("null argument");
    const adaptcore_status rc = adapter_size(M, N, K, AC_BF16_BF16OUT, 0, adapters, rank);
    if (rc != AC_OK) return rc;
    std::string out;
    if (M > 0 && N > 0) {
      const bool low_rank = adapters > 0 && rank > 0;
      const AdapterWay w = adapter_way(M, N, K, low_rank ? rank : 0, true);
      if (low_rank && !w.beside) out += "k_shrink;";
      out += (w.fused ? "k_adapter" : w.beside ? "k_multi_shrink" : "k_multi") + name(w.how->tile);
      if (w.how->pk > 1) out += " x" + std::to_string(w.how->pk);
      if (!w.fused) out += ";k_adapter_sum";
    }
    if ((int64_t)out.size() + 1 > len) return invalid("buffer too small");
    std::memcpy(buf, out.c_str(), out.size() + 1);
    return AC_OK;
  });
}

adaptcore_status adaptcore_gated_ffn_kernels(int64_t M, int64_t D, int64_t F, uint32_t layouts, int32_t backward,
                                             char* buf, int64_t len) {
  return guarded([&] {
    if (!buf || len < 1) return invalid("null argument");
    const FfnSize z = {M, D, F, AC_TYPE_BF16, layouts, AC_ACT_SILU};
    const adaptcore_status rc = ffn_check(z, AC_FFN_UP_COL | AC_FFN_DOWN_COL);
    if (rc != AC_OK) return rc;
    std::string out;
    auto add = [&](const FfnChoice& c, const char* fused, const char* sum) {
      out += (out.empty() ? "" : ";") + std::string(c.fused ? fused : "k_multi") + name(c.tile);
      if (c.pk > 1) out += " x" + std::to_string(c.pk);
      if (!c.fused && (c.pk > 1 || fused[0])) out += std::string(";") + sum;
    };
    const int kd = (int)cdiv(D, 64), kf = (int)cdiv(F, 64), km = (int)cdiv(M, 64);
    const bool direct = D % 8 == 0 && (z.up_col() || F % 8 == 0);
    if (!backward) {
      if (M == 0 || F == 0)
        out = "";
      else if (rows_kernel(M, F, D, 2, z.up_col(), direct))
        out = "k_rows<" + std::to_string(M <= 16 ? 1 : 2) + ">";
      else if (plain_projections(z, direct))
        out = "product;product;k_gated_sum";
      else
        add(ffn_choice(z.up_col() ? FFN_GATED : FFN_GATED_ROWS, M, 2 * F, D, kd), "k_gated", "k_gated_sum");
    } else if (D > 0) {
      if (M > 0 && F > 0) add(ffn_choice(FFN_DGATE, M, F, D, kd), "k_dgate", "k_dgate_sum");
      if (M > 0) add(ffn_choice(FFN_DX, M, D, 2 * F, 2 * kf), "", "k_plain_sum");
      if (F > 0) add(ffn_choice(FFN_DW, 3 * F, D, M, km), "", "k_plain_sum");
    }
    if ((int64_t)out.size() + 1 > len) return invalid("buffer too small");
    std::memcpy(buf, out.c_str(), out.size() + 1);
    return AC_OK;
  });
}

adaptcore_status adaptcore_layer_norm(int64_t rows, int64_t cols, int32_t type, int32_t weight_type, const void* X,
                                      int64_t ldx, const void* weight, const void* bias, float eps, void* Y,
                                      int64_t ldy, float* mean, float* rstd, void* stream) {
  return guarded([&] {
    adaptcore_status st = norm_size(rows, cols);
    if (st == AC_OK) st = norm_types(type, weight_type);
    if (st != AC_OK) return st;
    const int64_t need = std::max<int64_t>(1, cols);
    if (ldx < need || ldy < need) return invalid("row pitch smaller than the row");
    if (!std::isfinite(eps) || eps < 0) return invalid("eps must be finite and not negative");
    if (rows == 0 || cols == 0) return AC_OK;
    if (!X || !Y) return invalid("null matrix pointer");
    const int e = type_bytes(type), w = type_bytes(weight_type);
    if (misaligned(X, e) || misaligned(Y, e) || misaligned(weight, w) || misaligned(bias, w) || misaligned(mean, 4) ||
        misaligned(rstd, 4))
      return invalid("pointer not aligned to its element size");
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const ac::NormArgs a = {X, ldx, weight, bias, Y, ldy, mean, rstd, rows, cols, eps};
    return launched(
        ac::launch_norm(a, type, weight_type, ac::op_compute_units(), static_cast<hipStream_t>(stream)), 1);
  });
}

adaptcore_status adaptcore_layer_norm_backward(int64_t rows, int64_t cols, int32_t type, int32_t weight_type,
                                               const void* dY, int64_t lddy, const void* X, int64_t ldx,
                                               const void* weight, const float* mean, const float* rstd, void* dX,
                                               int64_t lddx, void* dweight, void* dbias, void* stream) {
  return guarded([&] {
    adaptcore_status st = norm_size(rows, cols);
    if (st == AC_OK) st = norm_types(type, weight_type);
    if (st != AC_OK) return st;
    const int64_t need = std::max<int64_t>(1, cols);
    if (lddy < need || ldx < need || lddx < need) return invalid("row pitch smaller than the row");
    if (cols == 0 || (rows == 0 && !dweight && !dbias)) return AC_OK;
    if (rows > 0 && (!dY || !X || !dX || !mean || !rstd)) return invalid("null pointer");
    const int e = type_bytes(type), w = type_bytes(weight_type);
    if (misaligned(dY, e) || misaligned(X, e) || misaligned(dX, e) || misaligned(weight, w) ||
        misaligned(dweight, w) || misaligned(dbias, w) || misaligned(mean, 4) || misaligned(rstd, 4))
      return invalid("pointer not aligned to its element size");
    st = ac::op_ready();
    if (st != AC_OK) return st;
    const int n_cu = ac::op_compute_units();
    ac::NormBwdArgs a = {dY, lddy, X, ldx, weight, mean, rstd, dX, lddx, dweight, dbias, rows, cols, nullptr, 0};
    a.parts = ac::norm_bwd_parts(a, n_cu);
    std::unique_lock<std::mutex> hold;
    if (a.parts > 0) {
      char* ws = nullptr;
      st = ac::op_workspace(static_cast<hipStream_t>(stream), (int64_t)a.parts * 2 * cols * 4, &ws, &hold);
      if (st != AC_OK) return st;
      a.part = reinterpret_cast<float*>(ws);
    }
    int n = 0;
    const hipError_t err =
        ac::launch_norm_bwd(a, type, weight_type, n_cu, static_cast<hipStream_t>(stream), &n);
    return launched(err, n);
  });
}

int64_t adaptcore_layer_norm_backward_workspace(int64_t rows, int64_t cols) {
  int64_t bytes = 0;
  const adaptcore_status st = guarded([&] {
    const adaptcore_status rc = norm_size(rows, cols);
    if (rc != AC_OK) return rc;
    ac::NormBwdArgs a;
    std::memset(&a, 0, sizeof a);
    a.rows = rows;
    a.cols = cols;
    a.dw = &bytes;  // any address: wanted
    if (cols > 0) bytes = (int64_t)ac::norm_bwd_parts(a, ac::op_compute_units()) * 2 * cols * 4;
    return AC_OK;
  });
  return st == AC_OK ? bytes : (int64_t)st;
}

}  // extern "C"
