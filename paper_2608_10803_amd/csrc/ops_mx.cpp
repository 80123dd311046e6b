// C entry points of the microscaled 4-bit matrices: checks, workspace, choice
// of kernels, launches.
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

// Counts the workspace, or (s->base) launches.
adaptcore_status run_mx(MxCall c, Scratch* s, hipStream_t st, int* launches) {
  const bool run = s->base != nullptr;
  hipError_t e = hipSuccess;
  if (c.a_type != AC_TYPE_MXFP4 && c.K > 0) {
    ac::MxQuantArgs q = {c.A, c.lda, c.M, c.K, nullptr, 16 * blocks_of(c.K), nullptr, (blocks_of(c.K) + 3) / 4 * 4};
    q.codes = s->take<uint8_t>(c.M * q.ld);
    q.scales = s->take<uint8_t>(c.M * q.lds);
    c.p.a = {q.codes, q.ld, q.scales, q.lds};
    if (run) e = ac::launch_mx_quantize(q, c.a_type, false, st);
    ++*launches;
  }
  if (run && e == hipSuccess) e = ac::launch_mx_rows(c.p, c.gated, st);
  ++*launches;
  return launched(e, 0);
}

adaptcore_status product(MxCall c, hipStream_t s) {
  adaptcore_status st = check_call(&c);
  if (st != AC_OK || c.M == 0 || c.N == 0) return st;
  st = ac::op_ready();
  if (st != AC_OK) return st;
  return with_scratch(s, [&](Scratch* w, int* n) { return run_mx(c, w, s, n); });
}

}  // namespace

extern "C" {

adaptcore_status adaptcore_mxfp4_quantize(int64_t rows, int64_t cols, int32_t type, uint32_t layout, const void* X,
                                          int64_t ldx, uint8_t* codes, int64_t ld_codes, uint8_t* scales,
                                          int64_t ld_scales, void* stream) {
  return guarded([&] {
    if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 31))
      return invalid("rows and cols must be in [0, 2^31)");
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
    const ac::MxQuantArgs a = {X, ldx, rows, cols, codes, ld_codes, scales, ld_scales};
    const hipError_t e = ac::launch_mx_quantize(a, type, col, static_cast<hipStream_t>(stream));
    if (e == hipErrorInvalidValue) return unsupported("launch grid too large");
    return launched(e, 1);
  });
}

adaptcore_status adaptcore_mxfp4_dequantize(int64_t rows, int64_t cols, int32_t type, const uint8_t* codes,
                                            int64_t ld_codes, const uint8_t* scales, int64_t ld_scales, void* Y,
                                            int64_t ldy, void* stream) {
  return guarded([&] {
    if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 31))
      return invalid("rows and cols must be in [0, 2^31)");
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
    MxCall c = {};
    c.M = M;
    c.N = N;
    c.K = K;
    c.gated = gated != 0;
    c.p.blocks = (int)blocks_of(K);
    Scratch s;
    int n = 0;
    rc = run_mx(c, &s, nullptr, &n);
    bytes = s.used;
    return rc;
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
      if (a_type != AC_TYPE_MXFP4 && K > 0) out = "k_mx_quant;";
      out += "k_mx_rows";
    }
    if ((int64_t)out.size() + 1 > len) return invalid("buffer too small");
    std::memcpy(buf, out.c_str(), out.size() + 1);
    return AC_OK;
  });
}

}  // extern "C"
