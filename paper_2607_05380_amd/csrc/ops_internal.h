// Launch interface between the host entry points of the student's operators
// (ops.cpp) and their kernels (kernels_rows.hip, kernels_block.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tabpack {

int set_error(int code, const char* msg);

constexpr int kRowMaxCols = 32768;   // widest row that the row kernels hold in registers
constexpr int kDistillMaxK = 256;    // teacher entries per row

// One pass over rows: v = x (+ residual); NORM: y = v rho w; QUANT: 8-bit codes
// and a scale per row of v or y.
struct RowArgs {
  const void* x;
  const void* residual;   // or NULL
  const float* weight;    // [cols] (norm)
  void* sum;              // or NULL: v in the input type
  void* out;              // y in the input type (norm without codes)
  int8_t* q;              // codes
  float* scale;           // [rows]
  float* rstd;            // [rows] or NULL: rho
  int64_t rows, ldx, ldr, lds, ldo;
  int32_t cols;
  float eps;
};
enum RowMode { ROW_NORM = 0, ROW_NORM_Q8 = 1, ROW_Q8 = 2 };
hipError_t launch_rows(int prec, RowMode mode, const RowArgs& a, hipStream_t s);

struct NormBwdArgs {
  const void* sum;
  const void* dy;
  const void* dsum;       // or NULL
  const float* weight;
  const float* rstd;
  void* dx;
  float* dweight;         // [cols]
  float* partial;         // [norm_bwd_blocks(rows, cols), cols]
  int64_t rows, lds, ldy, ldd, ldx;
  int32_t cols;
};
int norm_bwd_blocks(int64_t rows, int32_t cols);
hipError_t launch_norm_bwd(int prec, const NormBwdArgs& a, hipStream_t s);

struct DistillArgs {
  const void* logits;
  const int32_t* idx;     // [rows, k]
  const float* teacher;   // [rows, k]
  const float* weight;    // [rows] or NULL: 1
  float* loss;            // [rows]
  void* grad;             // or NULL
  int64_t rows, ldz, ldg;
  int32_t classes, k;
  float tau;
};
hipError_t launch_distill(int prec, const DistillArgs& a, hipStream_t s);

// A matrix product C[m, n] = sum_k A(m, k) B(n, k) with an epilogue per element.
enum MmType { MM_BF16 = 0, MM_FP32 = 1, MM_I8 = 2 };
// How an operand lies in memory: depth-contiguous (element (r, k) at P[r * ld + k])
// or rows-contiguous (at P[k * ld + r]).
enum MmEpi {
  MM_PLAIN = 0,     // out = C (+ add)
  MM_GATE = 1,      // B holds n gate rows, then n up rows: out = act(C_gate) C_up; both to `pre` if given
  MM_GATE_BWD = 2,  // C = dh: out = [dh u act'(g) | dh act(g)], g and u from `pre`
  MM_Q8 = 3,        // out = C row_scale col_scale (+ bias)
  MM_Q8_GATE = 4,   // the same for 2 n columns, then act(gate) up
};
struct MmArgs {
  const void* A;
  const void* B;
  int64_t lda, ldb;
  int32_t M, N, K;        // N: output columns (gated: of each half)
  int32_t a_rmaj, b_rmaj; // 1: rows-contiguous
  // 1: zeros follow each of the operand's rows in memory up to a multiple of 16 bytes
  int32_t a_zero, b_zero;
  int32_t pad;            // MM_GATE, MM_GATE_BWD: columns behind each row of out that are set to zero (bf16, fp32)
  int32_t epi, act;
  const void* add;        // MM_PLAIN: or NULL
  float* pre;             // [M, 2N] gate and up values (MM_GATE: or NULL)
  void* out;
  int64_t ldadd, ldpre, ldo;
  const float* row_scale;
  const float* col_scale; // [N] or [2N]
  const float* bias;      // [N] or [2N], or NULL
  int32_t out_f32;        // MM_Q8*: type of out (elsewhere the operands')
  float* work;            // aligned copies of operands, partial sums of a split depth
  size_t work_bytes;
  // filled in by launch_mm
  int32_t tiles_m, tiles_n, splits, steps_per_split;
};
// Bytes of `work` that the product needs (0: none).
size_t mm_workspace(MmType type, const MmArgs& a);
hipError_t launch_mm(MmType type, const MmArgs& a, hipStream_t s);
// Two independent products of one type, a with depth-contiguous A and
// rows-contiguous B (MM_PLAIN or MM_GATE_BWD), b with rows-contiguous operands
// (MM_PLAIN), of the same matrix A and the same work: in one launch where that is
// faster.
// One whose out is NULL is left out; the other's result does not depend on it.
size_t mm_pair_workspace(MmType type, const MmArgs& a, const MmArgs& b);
hipError_t launch_mm_pair(MmType type, const MmArgs& a, const MmArgs& b, hipStream_t s);

}  // namespace tabpack
