// C entry points of the joint between a block and the residual stream: checks,
// workspace, launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "ops.h"
#include "ops_host.h"

namespace {

using namespace ac::host;

adaptcore_status join_size(int64_t rows, int64_t cols, int64_t gate_rows) {
  if (rows < 0 || rows >= (1LL << 31) || cols < 0 || cols >= (1LL << 30))
    return invalid("rows must be in [0, 2^31) and cols in [0, 2^30)");
  if (gate_rows < 0 || gate_rows >= (1LL << 31) || (gate_rows > 0 && rows % gate_rows != 0))
    return invalid("the gate's rows must divide the rows");
  return AC_OK;
}

adaptcore_status pitch(const void* p, int64_t ld, int64_t cols, int bytes) {
  if (ld < std::max<int64_t>(1, cols)) return invalid("row pitch smaller than the row");
  if (misaligned(p, bytes)) return invalid("pointer not aligned to its element size");
  return AC_OK;
}

// Whether an output starts where an input or another output does. (Long and short
// rows are read again after parts of dX, dY and dgate are written, and lanes of any row
// share elements of their neighbours.)
bool over_another(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (auto o = outputs.begin(); o != outputs.end(); ++o)
    if (*o && (std::find(inputs.begin(), inputs.end(), *o) != inputs.end() || std::find(o + 1, outputs.end(), *o) != outputs.end()))
      return true;
  return false;
}

// Checks what both passes share and fills the launch arguments.
adaptcore_status join_args(const adaptcore_residual_norm_t* p, ac::JoinArgs* a) {
  if (!p) return invalid("null argument");
  adaptcore_status st = join_size(p->rows, p->cols, p->gate ? p->gate_rows : 0);
  if (st != AC_OK) return st;
  if (p->gate && p->gate_rows < 1) return invalid("the gate's rows must divide the rows");
  if (p->type != AC_TYPE_F32 && p->type != AC_TYPE_BF16 && p->type != AC_TYPE_F16)
    return unsupported("unknown element type");
  if (p->residual_type != AC_TYPE_F32 && p->residual_type != p->type)
    return unsupported("the residual stream must be fp32 or of the block's type");
  if (p->weight_type != AC_TYPE_F32 && p->weight_type != p->type)
    return unsupported("the weights must be fp32 or of the block's type");
  if (p->norm != AC_NORM_RMS && p->norm != AC_NORM_LAYER) return unsupported("unknown norm");
  if (!std::isfinite(p->eps) || p->eps < 0) return invalid("eps must be finite and not negative");
  if (!std::isfinite(p->scale)) return invalid("scale must be finite");
  const int rb = type_bytes(p->residual_type), b = type_bytes(p->type), w = type_bytes(p->weight_type);
  const bool some = p->rows > 0 && p->cols > 0;
  if (some && !p->Y && (p->post || p->gate)) return invalid("a norm after the block or a gate needs Y");
  if (!p->post && (p->post_weight || p->post_bias)) return invalid("weights of a norm that is not there");
  if (!p->pre && (p->weight || p->bias)) return invalid("weights of a norm that is not there");
  if (some && !p->X) return invalid("null matrix pointer");
  st = first_bad({pitch(p->X, p->ldx, p->cols, rb), p->Y ? pitch(p->Y, p->ldy, p->cols, b) : AC_OK,
                  p->gate ? pitch(p->gate, p->ld_gate, p->cols, w) : AC_OK, pitch(p->post_weight, 1, 1, w),
                  pitch(p->post_bias, 1, 1, w), pitch(p->weight, 1, 1, w), pitch(p->bias, 1, 1, w)});
  if (st != AC_OK) return st;
  std::memset(a, 0, sizeof *a);
  a->x = p->X;
  a->ldx = p->ldx;
  a->y = p->Y;
  a->ldy = p->ldy;
  a->w1 = p->post_weight;
  a->b1 = p->post_bias;
  a->gate = p->gate;
  a->ld_gate = p->ld_gate;
  a->per = p->gate ? p->rows / p->gate_rows : p->rows;
  a->w2 = p->weight;
  a->b2 = p->bias;
  a->rows = p->rows;
  a->cols = p->cols;
  a->scale = p->scale;
  a->eps = p->eps;
  a->layer = p->norm == AC_NORM_LAYER;
  a->post = p->post != 0;
  a->pre = p->pre != 0;
  return AC_OK;
}

// Pieces of a backward call's workspace.
void join_bwd_space(ac::JoinBwdArgs* b, Scratch* s) {
  ac::join_bwd_plan(b, ac::op_compute_units());
  b->part = b->sections > 0 && b->parts > 0 ? s->take<float>((int64_t)b->parts * b->sections * b->j.cols) : nullptr;
  const bool columns = b->sections > 0 || b->grad[4];
  b->means = columns && ac::join_bwd_means(b->j.cols) && b->j.rows > 0 ? s->take<float>(2 * b->j.rows) : nullptr;
}

}  // namespace

extern "C" {

adaptcore_status adaptcore_residual_norm(const adaptcore_residual_norm_t* p, void* R, int64_t ldr, void* N, int64_t ldn,
                                         uint8_t* codes, int64_t ld_codes, uint8_t* scales, int64_t ld_scales,
                                         float* stats, void* stream) {
  return guarded([&] {
    ac::JoinArgs a;
    adaptcore_status st = join_args(p, &a);
    if (st != AC_OK) return st;
    const int64_t blocks = cdiv(p->cols, 32);
    if (!a.pre && (N || codes)) return invalid("N needs its norm");
    const bool some = p->rows > 0 && p->cols > 0;
    if (some && (a.pre ? !N && !codes : !R)) return invalid("null matrix pointer");
    if ((codes == nullptr) != (scales == nullptr)) return invalid("codes and scales must both be given or both be null");
    st = first_bad({R ? pitch(R, ldr, p->cols, type_bytes(p->residual_type)) : AC_OK,
                    N ? pitch(N, ldn, p->cols, type_bytes(p->type)) : AC_OK, pitch(stats, 1, 1, 4)});
    if (st != AC_OK) return st;
    if (codes && (ld_codes < std::max<int64_t>(1, 16 * blocks) || ld_scales < std::max<int64_t>(1, blocks)))
      return invalid("pitch of codes or scales smaller than the row");
    if (!some) return AC_OK;
    st = ac::op_ready();
    if (st != AC_OK) return st;
    a.r = R;
    a.ldr = ldr;
    a.n = N;
    a.ldn = ldn;
    a.codes = codes;
    a.ld_codes = ld_codes;
    a.scales = scales;
    a.ld_scales = ld_scales;
    a.stats = stats;
    return launched(ac::launch_join(a, p->residual_type, p->type, p->weight_type, ac::op_compute_units(),
                                    static_cast<hipStream_t>(stream)),
                    1);
  });
}

adaptcore_status adaptcore_residual_norm_backward(const adaptcore_residual_norm_t* p, const void* dR, int64_t lddr,
                                                  const void* dN, int64_t lddn, const float* stats, void* dX,
                                                  int64_t lddx, void* dY, int64_t lddy, void* dpost_weight,
                                                  void* dpost_bias, void* dgate, int64_t ld_dgate, void* dweight,
                                                  void* dbias, void* stream) {
  return guarded([&] {
    ac::JoinBwdArgs b;
    std::memset(&b, 0, sizeof b);
    adaptcore_status st = join_args(p, &b.j);
    if (st != AC_OK) return st;
    const ac::JoinArgs& a = b.j;
    const int rb = type_bytes(p->residual_type), e = type_bytes(p->type), w = type_bytes(p->weight_type);
    if (!a.pre && (dN || dweight || dbias)) return invalid("gradients of a norm that is not there");
    if (!a.post && (dpost_weight || dpost_bias)) return invalid("gradients of a norm that is not there");
    if (!p->gate && dgate) return invalid("the gradient of a gate that is not there");
    if (p->rows > 0 && !p->Y && dY) return invalid("the gradient of a Y that is not there");
    if (p->rows > 0 && !dN && (dweight || dbias)) return invalid("the norm's gradients need dN");
    st = first_bad({dR ? pitch(dR, lddr, p->cols, rb) : AC_OK, dN ? pitch(dN, lddn, p->cols, e) : AC_OK,
                    dX ? pitch(dX, lddx, p->cols, rb) : AC_OK, dY ? pitch(dY, lddy, p->cols, e) : AC_OK,
                    dgate ? pitch(dgate, ld_dgate, p->cols, w) : AC_OK, pitch(dpost_weight, 1, 1, w),
                    pitch(dpost_bias, 1, 1, w), pitch(dweight, 1, 1, w), pitch(dbias, 1, 1, w), pitch(stats, 1, 1, 4)});
    if (st != AC_OK) return st;
    const bool sums = dpost_weight || dpost_bias || dweight || dbias || dgate;
    if (p->cols == 0 || (!sums && !dX && !dY) || (p->rows == 0 && !sums)) return AC_OK;
    if (p->rows > 0 && !dR && !dN) return invalid("dR or dN is needed");
    if (p->rows > 0 && !stats && (a.post || dN)) return invalid("the forward pass's statistics are needed");
    if (p->rows > 0 && over_another({dX, dY, dgate}, {dR, dN, p->X, p->Y, p->gate}))
      return invalid("dX, dY and dgate must not lie over an input or each other");
    st = ac::op_ready();
    if (st != AC_OK) return st;
    b.j.stats = const_cast<float*>(stats);
    b.dr = dR;
    b.lddr = lddr;
    b.dn = dN;
    b.lddn = lddn;
    b.dx = dX;
    b.lddx = lddx;
    b.dy = dY;
    b.lddy = lddy;
    void* const grads[5] = {dpost_weight, dpost_bias, dweight, dbias, dgate};
    std::memcpy(b.grad, grads, sizeof grads);
    b.ld_dgate = ld_dgate;
    b.gate_rows = p->gate ? p->gate_rows : 0;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return with_scratch(s, [&](Scratch* ws, int* n) {
      join_bwd_space(&b, ws);
      if (!ws->base) return AC_OK;
      return launched(
          ac::launch_join_bwd(b, p->residual_type, p->type, p->weight_type, ac::op_compute_units(), s, n), 0);
    });
  });
}

int64_t adaptcore_residual_norm_backward_workspace(int64_t rows, int64_t cols, int64_t gate_rows) {
  int64_t bytes = 0;
  const adaptcore_status st = guarded([&] {
    const adaptcore_status rc = join_size(rows, cols, gate_rows);
    if (rc != AC_OK || rows == 0 || cols == 0) return rc;
    for (bool gated : {false, true}) {
      if (gated && gate_rows == 0) continue;
      ac::JoinBwdArgs b;
      std::memset(&b, 0, sizeof b);
      b.j.rows = rows;
      b.j.cols = cols;
      b.j.per = gate_rows > 0 ? rows / gate_rows : rows;
      b.gate_rows = gate_rows;
      for (int k = 0; k < (gated ? 5 : 4); ++k) b.grad[k] = &bytes;  // any address: wanted
      Scratch s;
      join_bwd_space(&b, &s);
      bytes = std::max(bytes, s.used);
    }
    return AC_OK;
  });
  return st == AC_OK ? bytes : (int64_t)st;
}

}  // extern "C"
