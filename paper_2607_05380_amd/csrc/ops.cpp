// Entry points of the student network's operators (include/tabpack.h):
// argument checks, then one launch function of the kernels' files.
#include <algorithm>
#include <cfloat>
#include <cstdarg>
#include <cstdio>

#include "../../include/tabpack.h"
#include "ops_internal.h"

using namespace tabpack;

namespace {

static_assert(kRowMaxCols == PACK_ROW_MAX_COLS && kDistillMaxK == PACK_DISTILL_MAX_K, "the header's limits");

int bad(const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_error(PACK_EINVAL, buf);
}

int done(const char* what, hipError_t e) {
  if (e == hipSuccess) return PACK_OK;
  if (e == hipErrorInvalidConfiguration) return bad("%s: more tiles than a launch holds", what);
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return set_error(PACK_EHIP, buf);
}

constexpr int64_t kMaxExtent = 0x7fffffff;  // rows, leading dimensions

bool known(int32_t precision) { return precision == PACK_PREC_BF16 || precision == PACK_PREC_FP32; }

// A leading dimension that fits rows of `cols` elements.
bool ld_ok(int64_t ld, int64_t cols) { return ld >= cols && ld <= kMaxExtent; }

bool aligned(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

int check_rows(int32_t precision, int64_t rows, int32_t cols) {
  if (!known(precision)) return bad("unknown precision %d", precision);
  if (rows < 0 || rows > kMaxExtent) return bad("rows=%lld out of [0, 2^31 - 1]", (long long)rows);
  if (cols < 1 || cols > kRowMaxCols) return bad("cols=%d out of [1, %d]", cols, kRowMaxCols);
  return PACK_OK;
}

int norm_rows(RowMode mode, RowArgs& a, int32_t precision, hipStream_t stream) {
  const int rc = check_rows(precision, a.rows, a.cols);
  if (rc != PACK_OK) return rc;
  if (mode != ROW_Q8 && !(a.eps >= 0.0f && a.eps <= FLT_MAX)) return bad("eps must be finite and not negative");
  if (!ld_ok(a.ldx, a.cols) || (a.residual && !ld_ok(a.ldr, a.cols)) || (a.sum && !ld_ok(a.lds, a.cols)) ||
      !ld_ok(a.ldo, a.cols))
    return bad("a leading dimension is smaller than cols=%d or too large", a.cols);
  if (a.rows == 0) return PACK_OK;
  if (!a.x || (mode != ROW_Q8 && !a.weight) || (mode == ROW_NORM ? !a.out : !a.q || !a.scale))
    return bad("NULL device pointer");
  return done("row kernel", launch_rows(precision, mode, a, stream));
}

constexpr int32_t kMaxWidth = 1 << 24;  // d_in, hidden, d_out, outputs

bool known_act(int32_t act) { return act >= PACK_ACT_SILU && act <= PACK_ACT_RELU; }

MmType type_of(int32_t precision) { return precision == PACK_PREC_BF16 ? MM_BF16 : MM_FP32; }

// The products of a gated block (x [T, D], hidden width F, y [T, O]).
// (h and [dg | du] in rows of ff_ld() elements, zeros behind their ends)
int64_t ff_ld(MmType t, int64_t cols) { return PACK_FF_LD(t == MM_BF16 ? PACK_PREC_BF16 : PACK_PREC_FP32, cols); }
MmArgs mm_gate(MmType t, int64_t T, int32_t D, int32_t F) {
  MmArgs a{};
  a.M = (int32_t)T, a.N = F, a.K = D, a.epi = MM_GATE, a.ldo = ff_ld(t, F), a.pad = (int32_t)(a.ldo - F);
  return a;
}
MmArgs mm_down(MmType t, int64_t T, int32_t F, int32_t O) {
  MmArgs a{};
  a.M = (int32_t)T, a.N = O, a.K = F, a.epi = MM_PLAIN, a.lda = ff_ld(t, F), a.a_zero = 1;
  return a;
}
MmArgs mm_dh(MmType t, int64_t T, int32_t F, int32_t O) {
  MmArgs a{};
  a.M = (int32_t)T, a.N = F, a.K = O, a.b_rmaj = 1, a.epi = MM_GATE_BWD;
  a.ldo = ff_ld(t, 2 * (int64_t)F), a.pad = (int32_t)(a.ldo - 2 * (int64_t)F);
  return a;
}
MmArgs mm_dx(MmType t, int64_t T, int32_t D, int32_t F) {
  MmArgs a{};
  a.M = (int32_t)T, a.N = D, a.K = 2 * F, a.b_rmaj = 1, a.epi = MM_PLAIN;
  a.lda = ff_ld(t, 2 * (int64_t)F), a.a_zero = 1;
  return a;
}
MmArgs mm_dwd(MmType t, int64_t T, int32_t F, int32_t O) {
  MmArgs a{};
  a.M = O, a.N = F, a.K = (int32_t)T, a.a_rmaj = a.b_rmaj = 1, a.epi = MM_PLAIN, a.ldb = ff_ld(t, F), a.b_zero = 1;
  return a;
}
MmArgs mm_dwg(MmType t, int64_t T, int32_t D, int32_t F) {
  MmArgs a{};
  a.M = 2 * F, a.N = D, a.K = (int32_t)T, a.a_rmaj = a.b_rmaj = 1, a.epi = MM_PLAIN;
  a.lda = ff_ld(t, 2 * (int64_t)F), a.a_zero = 1;
  return a;
}
MmArgs mm_q8(int64_t rows, int32_t outputs, int32_t depth, int32_t gate) {
  MmArgs a{};
  a.M = (int32_t)rows, a.N = outputs, a.K = depth, a.epi = gate < 0 ? MM_Q8 : MM_Q8_GATE, a.act = gate < 0 ? 0 : gate;
  return a;
}

int check_ff(int32_t precision, int32_t act, int64_t T, int32_t D, int32_t F, int32_t O) {
  if (!known(precision)) return bad("unknown precision %d", precision);
  if (!known_act(act)) return bad("unknown activation %d", act);
  if (T < 0 || T > kMaxExtent) return bad("tokens=%lld out of [0, 2^31 - 1]", (long long)T);
  if (D < 1 || F < 1 || O < 1 || D > kMaxWidth || F > kMaxWidth || O > kMaxWidth)
    return bad("d_in=%d, hidden=%d and d_out=%d must lie in [1, 2^24]", D, F, O);
  return PACK_OK;
}

int check_q8(int64_t rows, int32_t outputs, int32_t depth, int32_t gate) {
  if (gate != -1 && !known_act(gate)) return bad("unknown gate %d", gate);
  if (rows < 0 || rows > kMaxExtent) return bad("rows=%lld out of [0, 2^31 - 1]", (long long)rows);
  if (outputs < 1 || outputs > kMaxWidth) return bad("outputs=%d out of [1, 2^24]", outputs);
  if (depth < 1 || depth > PACK_Q8_MAX_DEPTH) return bad("depth=%d out of [1, %d]", depth, PACK_Q8_MAX_DEPTH);
  return PACK_OK;
}

int check_work(const void* work, size_t have, size_t need) {
  if (need == 0) return PACK_OK;
  if (!work) return bad("work is NULL");
  if (have < need) return bad("workspace has %zu bytes, %zu needed", have, need);
  if (!aligned(work, 16)) return bad("workspace must be 16-byte aligned");
  return PACK_OK;
}

}  // namespace

extern "C" {

int pack_gated_ff_workspace_size(int32_t precision, int64_t tokens, int32_t d_in, int32_t hidden, int32_t d_out,
                                 int32_t backward, size_t* bytes) {
  if (!bytes) return bad("bytes is NULL");
  const int rc = check_ff(precision, PACK_ACT_SILU, tokens, d_in, hidden, d_out);
  if (rc != PACK_OK) return rc;
  const MmType t = type_of(precision);
  if (!backward)
    *bytes = std::max(mm_workspace(t, mm_gate(t, tokens, d_in, hidden)),
                      mm_workspace(t, mm_down(t, tokens, hidden, d_out)));
  else
    *bytes = std::max(mm_pair_workspace(t, mm_dh(t, tokens, hidden, d_out), mm_dwd(t, tokens, hidden, d_out)),
                      mm_pair_workspace(t, mm_dx(t, tokens, d_in, hidden), mm_dwg(t, tokens, d_in, hidden)));
  return PACK_OK;
}

int pack_gated_ff_forward(const void* x, int64_t ldx, const void* w_gate_up, int64_t ldwg, const void* w_down,
                          int64_t ldwd, const void* residual, int64_t ldr, int32_t precision, int32_t act,
                          int64_t tokens, int32_t d_in, int32_t hidden, int32_t d_out, float* gate_up_out,
                          void* hidden_out, void* out, int64_t ldo, void* work, size_t work_bytes,
                          hipStream_t stream) {
  int rc = check_ff(precision, act, tokens, d_in, hidden, d_out);
  if (rc != PACK_OK) return rc;
  if (!ld_ok(ldx, d_in) || !ld_ok(ldwg, d_in) || !ld_ok(ldwd, hidden) || (residual && !ld_ok(ldr, d_out)) ||
      !ld_ok(ldo, d_out))
    return bad("a leading dimension is smaller than its matrix's rows or too large");
  if (tokens == 0) return PACK_OK;
  if (!x || !w_gate_up || !w_down || !hidden_out || !out) return bad("NULL device pointer");
  size_t need = 0;
  rc = pack_gated_ff_workspace_size(precision, tokens, d_in, hidden, d_out, 0, &need);
  if (rc == PACK_OK) rc = check_work(work, work_bytes, need);
  if (rc != PACK_OK) return rc;
  const MmType t = type_of(precision);
  MmArgs a = mm_gate(t, tokens, d_in, hidden);
  a.A = x, a.lda = ldx, a.B = w_gate_up, a.ldb = ldwg, a.act = act;
  a.pre = gate_up_out, a.ldpre = 2 * (int64_t)hidden, a.out = hidden_out;
  a.work = static_cast<float*>(work), a.work_bytes = work_bytes;
  rc = done("gate and up projections", launch_mm(t, a, stream));
  if (rc != PACK_OK) return rc;
  MmArgs d = mm_down(t, tokens, hidden, d_out);
  d.A = hidden_out, d.B = w_down, d.ldb = ldwd, d.add = residual, d.ldadd = ldr;
  d.out = out, d.ldo = ldo, d.work = a.work, d.work_bytes = work_bytes;
  return done("down projection", launch_mm(t, d, stream));
}

int pack_gated_ff_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w_gate_up,
                           int64_t ldwg, const void* w_down, int64_t ldwd, const float* gate_up, const void* hidden_in,
                           int32_t precision, int32_t act, int64_t tokens, int32_t d_in, int32_t hidden,
                           int32_t d_out, void* dgate_up, void* dx_out, int64_t lddx, void* dw_gate_up_out,
                           void* dw_down_out, void* work, size_t work_bytes, hipStream_t stream) {
  int rc = check_ff(precision, act, tokens, d_in, hidden, d_out);
  if (rc != PACK_OK) return rc;
  if (!ld_ok(lddy, d_out) || !ld_ok(ldx, d_in) || !ld_ok(ldwg, d_in) || !ld_ok(ldwd, hidden) ||
      (dx_out && !ld_ok(lddx, d_in)))
    return bad("a leading dimension is smaller than its matrix's rows or too large");
  if (tokens > 0 && (!dy || !x || !w_gate_up || !w_down || !gate_up || !hidden_in || !dgate_up))
    return bad("NULL device pointer");
  size_t need = 0;
  rc = pack_gated_ff_workspace_size(precision, tokens, d_in, hidden, d_out, 1, &need);
  if (rc == PACK_OK) rc = check_work(work, work_bytes, need);
  if (rc != PACK_OK) return rc;
  const MmType t = type_of(precision);
  // [dg | du] beside dw_down, then dx beside dw_gate_up
  MmArgs dh = mm_dh(t, tokens, hidden, d_out), dwd = mm_dwd(t, tokens, hidden, d_out);
  MmArgs dx = mm_dx(t, tokens, d_in, hidden), dwg = mm_dwg(t, tokens, d_in, hidden);
  dh.A = dy, dh.lda = lddy, dh.B = w_down, dh.ldb = ldwd, dh.act = act;
  dh.pre = const_cast<float*>(gate_up), dh.ldpre = 2 * (int64_t)hidden, dh.out = dgate_up;
  dwd.A = dy, dwd.lda = lddy, dwd.B = hidden_in, dwd.out = dw_down_out, dwd.ldo = hidden;
  dx.A = dgate_up, dx.B = w_gate_up, dx.ldb = ldwg, dx.out = dx_out, dx.ldo = lddx;
  dwg.A = dgate_up, dwg.B = x, dwg.ldb = ldx, dwg.out = dw_gate_up_out, dwg.ldo = d_in;
  for (MmArgs* a : {&dh, &dwd, &dx, &dwg}) a->work = static_cast<float*>(work), a->work_bytes = work_bytes;
  if (!dx_out && !dw_gate_up_out) dh.out = nullptr;
  hipError_t e = launch_mm_pair(t, dh, dwd, stream);
  if (e == hipSuccess) e = launch_mm_pair(t, dx, dwg, stream);
  return done("gated block backward", e);
}

int pack_q8_matmul_workspace_size(int64_t rows, int32_t outputs, int32_t depth, int32_t gate, size_t* bytes) {
  if (!bytes) return bad("bytes is NULL");
  const int rc = check_q8(rows, outputs, depth, gate);
  if (rc != PACK_OK) return rc;
  *bytes = mm_workspace(MM_I8, mm_q8(rows, outputs, depth, gate));
  return PACK_OK;
}

int pack_q8_matmul(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw,
                   const float* w_scale, const float* bias, int32_t gate, int32_t precision, int64_t rows,
                   int32_t outputs, int32_t depth, void* out, int64_t ldo, void* work, size_t work_bytes,
                   hipStream_t stream) {
  if (!known(precision)) return bad("unknown precision %d", precision);
  int rc = check_q8(rows, outputs, depth, gate);
  if (rc != PACK_OK) return rc;
  if (!ld_ok(ldx, depth) || !ld_ok(ldw, depth) || !ld_ok(ldo, outputs))
    return bad("a leading dimension is smaller than its matrix's rows or too large");
  if (rows == 0) return PACK_OK;
  if (!x || !x_scale || !w || !w_scale || !out) return bad("NULL device pointer");
  MmArgs a = mm_q8(rows, outputs, depth, gate);
  rc = check_work(work, work_bytes, mm_workspace(MM_I8, a));
  if (rc != PACK_OK) return rc;
  a.A = x, a.lda = ldx, a.B = w, a.ldb = ldw, a.row_scale = x_scale, a.col_scale = w_scale, a.bias = bias;
  a.out = out, a.ldo = ldo, a.out_f32 = precision == PACK_PREC_FP32;
  a.work = static_cast<float*>(work), a.work_bytes = work_bytes;
  return done("8-bit product", launch_mm(MM_I8, a, stream));
}

int pack_add_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight,
                      int32_t precision, int64_t rows, int32_t cols, float eps, void* sum_out, int64_t lds,
                      void* out, int64_t ldo, float* rstd_out, hipStream_t stream) {
  RowArgs a{};
  a.x = x, a.ldx = ldx, a.residual = residual, a.ldr = ldr, a.weight = weight;
  a.rows = rows, a.cols = cols, a.eps = eps;
  a.sum = sum_out, a.lds = lds, a.out = out, a.ldo = ldo, a.rstd = rstd_out;
  return norm_rows(ROW_NORM, a, precision, stream);
}

int pack_add_rms_norm_q8(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight,
                         int32_t precision, int64_t rows, int32_t cols, float eps, void* sum_out, int64_t lds,
                         int8_t* q_out, int64_t ldq, float* scale_out, hipStream_t stream) {
  RowArgs a{};
  a.x = x, a.ldx = ldx, a.residual = residual, a.ldr = ldr, a.weight = weight;
  a.rows = rows, a.cols = cols, a.eps = eps;
  a.sum = sum_out, a.lds = lds, a.q = q_out, a.ldo = ldq, a.scale = scale_out;
  return norm_rows(ROW_NORM_Q8, a, precision, stream);
}

int pack_quantize_rows(const void* x, int64_t ldx, int32_t precision, int64_t rows, int32_t cols, int8_t* q_out,
                       int64_t ldq, float* scale_out, hipStream_t stream) {
  RowArgs a{};
  a.x = x, a.ldx = ldx, a.rows = rows, a.cols = cols, a.q = q_out, a.ldo = ldq, a.scale = scale_out;
  return norm_rows(ROW_Q8, a, precision, stream);
}

int pack_rms_norm_backward_workspace_size(int64_t rows, int32_t cols, size_t* bytes) {
  if (!bytes) return bad("bytes is NULL");
  const int rc = check_rows(PACK_PREC_FP32, rows, cols);
  if (rc != PACK_OK) return rc;
  *bytes = (size_t)norm_bwd_blocks(rows, cols) * (size_t)cols * 4;
  return PACK_OK;
}

int pack_rms_norm_backward(const void* dy, int64_t ldy, const void* sum, int64_t lds, const float* weight,
                           const float* rstd, const void* dsum, int64_t ldd, int32_t precision, int64_t rows,
                           int32_t cols, void* dx_out, int64_t ldx, float* dweight_out, void* work,
                           size_t work_bytes, hipStream_t stream) {
  int rc = check_rows(precision, rows, cols);
  if (rc != PACK_OK) return rc;
  if (!ld_ok(ldy, cols) || !ld_ok(lds, cols) || (dsum && !ld_ok(ldd, cols)) || !ld_ok(ldx, cols))
    return bad("a leading dimension is smaller than cols=%d or too large", cols);
  size_t need = 0;
  rc = pack_rms_norm_backward_workspace_size(rows, cols, &need);
  if (rc != PACK_OK) return rc;
  if (!weight || !dweight_out || !work || (rows > 0 && (!dy || !sum || !rstd || !dx_out)))
    return bad("NULL device pointer");
  if (work_bytes < need) return bad("workspace has %zu bytes, %zu needed", work_bytes, need);
  if (!aligned(work, 4)) return bad("workspace must be 4-byte aligned");
  NormBwdArgs a{};
  a.sum = sum, a.lds = lds, a.dy = dy, a.ldy = ldy, a.dsum = dsum, a.ldd = ldd;
  a.weight = weight, a.rstd = rstd, a.dx = dx_out, a.ldx = ldx, a.dweight = dweight_out;
  a.partial = static_cast<float*>(work), a.rows = rows, a.cols = cols;
  return done("norm backward", launch_norm_bwd(precision, a, stream));
}

int pack_distill_topk(const void* logits, int64_t ldz, int32_t precision, int64_t rows, int32_t classes,
                      const int32_t* idx, const float* teacher, int32_t k, float temperature,
                      const float* row_weight, float* loss_out, void* grad_out, int64_t ldg, hipStream_t stream) {
  if (!known(precision)) return bad("unknown precision %d", precision);
  if (rows < 0 || rows > kMaxExtent) return bad("rows=%lld out of [0, 2^31 - 1]", (long long)rows);
  if (classes < 1) return bad("classes=%d must be positive", classes);
  if (k < 1 || k > kDistillMaxK) return bad("k=%d out of [1, %d]", k, kDistillMaxK);
  if (!(temperature >= FLT_MIN && temperature <= FLT_MAX && 1.0f / temperature >= FLT_MIN))
    return bad("temperature must be positive and finite");
  if (!ld_ok(ldz, classes) || (grad_out && !ld_ok(ldg, classes)))
    return bad("a leading dimension is smaller than classes=%d or too large", classes);
  if (rows == 0) return PACK_OK;
  if (!logits || !idx || !teacher || !loss_out) return bad("NULL device pointer");
  DistillArgs a{};
  a.logits = logits, a.ldz = ldz, a.idx = idx, a.teacher = teacher, a.weight = row_weight;
  a.loss = loss_out, a.grad = grad_out, a.ldg = ldg, a.rows = rows, a.classes = classes, a.k = k, a.tau = temperature;
  return done("distillation", launch_distill(precision, a, stream));
}

}  // extern "C"
