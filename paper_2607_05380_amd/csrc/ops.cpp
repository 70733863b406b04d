// Entry points of the student network's operators (include/tabpack.h):
// argument checks, then one launch function of the kernels' files.
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
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return set_error(PACK_EHIP, buf);
}

constexpr int64_t kMaxExtent = 0x7fffffff;  // rows, leading dimensions

bool known(int32_t precision) { return precision == PACK_PREC_BF16 || precision == PACK_PREC_FP32; }
int elem_size(int32_t precision) { return precision == PACK_PREC_BF16 ? 2 : 4; }

// A leading dimension that fits rows of `cols` elements.
bool ld_ok(int64_t ld, int64_t cols) { return ld >= cols && ld <= kMaxExtent; }

bool aligned(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

// Every row of the matrix starts at a multiple of `bytes`.
bool rows_aligned(const void* p, int64_t ld, int size, int bytes) {
  return aligned(p, bytes) && ld * size % bytes == 0;
}

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
  const int es = elem_size(precision), ve = 16 / es;
  a.vec = a.cols % ve == 0 && rows_aligned(a.x, a.ldx, es, 16) && (!a.residual || rows_aligned(a.residual, a.ldr, es, 16)) &&
          (!a.sum || rows_aligned(a.sum, a.lds, es, 16)) && (!a.weight || aligned(a.weight, 16)) &&
          (mode == ROW_NORM ? rows_aligned(a.out, a.ldo, es, 16) : rows_aligned(a.q, a.ldo, 1, ve));
  return done("row kernel", launch_rows(precision, mode, a, stream));
}

}  // namespace

extern "C" {

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
  const int es = elem_size(precision);
  NormBwdArgs a{};
  a.sum = sum, a.lds = lds, a.dy = dy, a.ldy = ldy, a.dsum = dsum, a.ldd = ldd;
  a.weight = weight, a.rstd = rstd, a.dx = dx_out, a.ldx = ldx, a.dweight = dweight_out;
  a.partial = static_cast<float*>(work), a.rows = rows, a.cols = cols;
  a.vec = cols % (16 / es) == 0 && rows_aligned(dy, ldy, es, 16) && rows_aligned(sum, lds, es, 16) &&
          (!dsum || rows_aligned(dsum, ldd, es, 16)) && rows_aligned(dx_out, ldx, es, 16) && aligned(weight, 16);
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
  const int es = elem_size(precision);
  DistillArgs a{};
  a.logits = logits, a.ldz = ldz, a.idx = idx, a.teacher = teacher, a.weight = row_weight;
  a.loss = loss_out, a.grad = grad_out, a.ldg = ldg, a.rows = rows, a.classes = classes, a.k = k, a.tau = temperature;
  a.vec = classes % (16 / es) == 0 && rows_aligned(logits, ldz, es, 16) &&
          (!grad_out || rows_aligned(grad_out, ldg, es, 16));
  return done("distillation", launch_distill(precision, a, stream));
}

}  // extern "C"
