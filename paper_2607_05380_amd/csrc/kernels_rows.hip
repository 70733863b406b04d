// Row kernels of the student network on gfx950: the root-mean-square norm with
// the residual's addition (forward, 8-bit output, backward), row quantisation,
// and distillation from a teacher's top logits.
//
// Each does a few operations a byte, so the bytes of one read and one write
// bound it.  A row is read once into the registers of the G threads that own
// it (16, 64, 256 or 1024, EPT elements each, by the row's length), reduced
// there, and written from there.  Thread t of a row owns the vectors t, t + G,
// t + 2G, ... of VE elements (16 bytes; VE = 1 where rows do not start at 16
// bytes or the length is no multiple of it), so a wave's accesses are
// contiguous.  Sums are held in fp32 and added in a fixed order.
#include "ops_internal.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// VE elements at p, as floats
template <int VE>
__device__ __forceinline__ void load_vec(const __bf16* p, float* v) {
  if constexpr (VE == 8) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, u[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
    }
  } else {
    static_assert(VE == 1);
    v[0] = (float)p[0];
  }
}
template <int VE>
__device__ __forceinline__ void load_vec(const float* p, float* v) {
  if constexpr (VE >= 4) {
#pragma unroll
    for (int i = 0; i < VE / 4; ++i) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * i + j] = u[j];
    }
  } else {
    static_assert(VE == 1);
    v[0] = p[0];
  }
}
template <int VE>
__device__ __forceinline__ void store_vec(__bf16* p, const float* v) {
  if constexpr (VE == 8) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x8*>(p) = o;
  } else {
    p[0] = (__bf16)v[0];
  }
}
template <int VE>
__device__ __forceinline__ void store_vec(float* p, const float* v) {
  if constexpr (VE == 4)
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  else
    p[0] = v[0];
}
// VE codes (whole numbers in [-127, 127])
template <int VE>
__device__ __forceinline__ void store_codes(int8_t* p, const float* v) {
  uint32_t w[VE >= 4 ? VE / 4 : 1];
  if constexpr (VE >= 4) {
#pragma unroll
    for (int i = 0; i < VE / 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i] |= ((uint32_t)(int32_t)v[4 * i + j] & 0xffu) << (8 * j);
    }
    if constexpr (VE == 8)
      *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
    else
      *reinterpret_cast<uint32_t*>(p) = w[0];
  } else {
    p[0] = (int8_t)(int32_t)v[0];
  }
}

struct OpAdd {
  __device__ static float op(float a, float b) { return a + b; }
  static constexpr float zero = 0.0f;
};
// Largest of values that are not negative; NaN counts as larger than infinity
// (the order of their bits), so it is not lost.
struct OpMaxMag {
  __device__ static float op(float a, float b) {
    return __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)));
  }
  static constexpr float zero = 0.0f;
};
struct OpMax {
  __device__ static float op(float a, float b) { return fmaxf(a, b); }
  static constexpr float zero = -__builtin_inff();
};

// Reduction over the G threads of a row; every one of them gets the result.
// G > 64: through LDS, one float per wave (`red`, 16 floats per use: a kernel
// gives each of its reductions its own, so one barrier serves).
template <int G, typename Op>
__device__ __forceinline__ float reduce_row(float v, float* red, int tid) {
#pragma unroll
  for (int m = (G < 64 ? G : 64) / 2; m >= 1; m >>= 1) v = Op::op(v, __shfl_xor(v, m, 64));
  if constexpr (G > 64) {
    if ((tid & 63) == 0) red[tid >> 6] = v;
    __syncthreads();
    float r = red[0];
#pragma unroll
    for (int w = 1; w < G / 64; ++w) r = Op::op(r, red[w]);
    v = r;
  }
  return v;
}

// 127 / a, 0 where a is 0 or so small that the quotient overflows (a row of
// such values has codes 0 and scale 0)
__device__ __forceinline__ float code_factor(float a) {
  const float f = 127.0f / a;
  return a > 0.0f && f < __builtin_inff() ? f : 0.0f;
}

// ------------------------------------------------- norm and quantisation --
// v = x (+ residual) in fp32; rho = (mean v^2 + eps)^(-1/2); y = v rho w.
// The codes of y are those of t = v w: rho > 0 is common to the row, so
// q = rint(t 127 / max|t|) and the scale is max|t| rho / 127 -- a row's codes
// do not depend on the order in which its squares were added.  A row that
// holds an infinity or NaN gets codes 0 and scale NaN.
template <typename T, int VE, int G, int EPT, int MODE>
__global__ __launch_bounds__(G > 256 ? G : 256) void rows_kernel(RowArgs a) {
  constexpr int NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE;
  __shared__ float red[2][2][16];
  const int tid = threadIdx.x, t = tid % G;
  static_assert(G <= 64 || RPB == 1, "a row's barriers are the block's");
  int turn = 0;  // rows take turns with two sets of LDS words: a row's barriers lie between their uses
  for (int64_t row = (int64_t)blockIdx.x * RPB + tid / G; row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    float v[EPT];
  #pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      if (c < a.cols) {
        load_vec<VE>(x + c, v + i * VE);
      } else {
  #pragma unroll
        for (int e = 0; e < VE; ++e) v[i * VE + e] = 0.0f;
      }
    }
    if (MODE != ROW_Q8 && a.residual) {
      const T* r = static_cast<const T*>(a.residual) + row * a.ldr;
      float u[EPT];
  #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        if (c < a.cols) load_vec<VE>(r + c, u + i * VE);
      }
  #pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((i * G + t) * VE < a.cols) {
  #pragma unroll
          for (int e = 0; e < VE; ++e) v[i * VE + e] += u[i * VE + e];
        }
    }
    float rho = 1.0f;
    if constexpr (MODE != ROW_Q8) {
      if (a.sum) {
        T* s = static_cast<T*>(a.sum) + row * a.lds;
  #pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VE;
          if (c < a.cols) store_vec<VE>(s + c, v + i * VE);
        }
      }
      float sq = 0.0f;
  #pragma unroll
      for (int e = 0; e < EPT; ++e) sq = fmaf(v[e], v[e], sq);
      sq = reduce_row<G, OpAdd>(sq, red[turn][0], tid);
      rho = 1.0f / sqrtf(sq / (float)a.cols + a.eps);
      if (a.rstd && t == 0) a.rstd[row] = rho;
  #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        if (c < a.cols) {
          float w[VE];
          load_vec<VE>(a.weight + c, w);
  #pragma unroll
          for (int e = 0; e < VE; ++e) v[i * VE + e] = MODE == ROW_NORM ? v[i * VE + e] * rho * w[e] : v[i * VE + e] * w[e];
        }
      }
    }
    if constexpr (MODE == ROW_NORM) {
      T* o = static_cast<T*>(a.out) + row * a.ldo;
  #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        if (c < a.cols) store_vec<VE>(o + c, v + i * VE);
      }
    } else {
      float m = 0.0f;
  #pragma unroll
      for (int e = 0; e < EPT; ++e) m = OpMaxMag::op(m, fabsf(v[e]));
      m = reduce_row<G, OpMaxMag>(m, red[turn][1], tid);
      const bool finite = m < __builtin_inff();
      const float f = finite ? code_factor(m) : 0.0f;
      if (t == 0) a.scale[row] = !finite ? __builtin_nanf("") : f == 0.0f ? 0.0f : m * rho / 127.0f;
      int8_t* q = a.q + row * a.ldo;
  #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        if (c < a.cols) {
          float k[VE];
  #pragma unroll
          for (int e = 0; e < VE; ++e) k[e] = finite ? rintf(v[i * VE + e] * f) : 0.0f;
          store_codes<VE>(q + c, k);
        }
      }
    }
  }
}

// --------------------------------------------------------- norm, backward --
// With g = w dy, rho as saved and D = cols:
//   dx = rho (g - v rho^2 / D sum_c g v) + dsum,   dweight = sum_rows dy v rho.
// A block walks over rows (gridDim apart) and keeps the columns' weight sums
// in registers; its sums go to one row of `partial`, which a second kernel
// adds up in order: no atomics, so the result does not change between runs.
template <typename T, int VE, int G, int EPT>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE;
  __shared__ float red[2][16];
  __shared__ float cols[RPB > 1 ? G * EPT : 1];
  const int tid = threadIdx.x, t = tid % G, rg = tid / G;
  float dw[EPT];
#pragma unroll
  for (int e = 0; e < EPT; ++e) dw[e] = 0.0f;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * RPB + rg; row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
    const T* s = static_cast<const T*>(a.sum) + row * a.lds;
    const T* dy = static_cast<const T*>(a.dy) + row * a.ldy;
    const float rho = a.rstd[row];
    float v[EPT], g[EPT];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      if (c < a.cols) {
        load_vec<VE>(s + c, v + i * VE);
        load_vec<VE>(dy + c, g + i * VE);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[i * VE + e] = g[i * VE + e] = 0.0f;
      }
    }
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      if (c < a.cols) {
        float w[VE];
        load_vec<VE>(a.weight + c, w);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          float& gg = g[i * VE + e];
          dw[i * VE + e] = fmaf(gg * v[i * VE + e], rho, dw[i * VE + e]);
          gg *= w[e];
          dot = fmaf(gg, v[i * VE + e], dot);
        }
      }
    }
    // (rows that span waves alternate between two sets of LDS words)
    dot = reduce_row<G, OpAdd>(dot, red[turn], tid);
    const float c1 = dot / (float)a.cols * rho * rho;
    T* dx = static_cast<T*>(a.dx) + row * a.ldx;
    const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.ldd : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      if (c < a.cols) {
        float o[VE];
        if (ds) {
          load_vec<VE>(ds + c, o);
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) o[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] = fmaf(rho, g[i * VE + e] - v[i * VE + e] * c1, o[e]);
        store_vec<VE>(dx + c, o);
      }
    }
  }
  // the block's sums: its row groups one after the other
  if constexpr (RPB > 1) {
    for (int r = 0; r < RPB; ++r) {
      if (rg == r) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const int c = (i * G + t) * VE + e;
            cols[c] = (r == 0 ? 0.0f : cols[c]) + dw[i * VE + e];
          }
      }
      __syncthreads();
    }
    for (int c = tid; c < a.cols; c += NT) a.partial[(int64_t)blockIdx.x * a.cols + c] = cols[c];
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int c = (i * G + t) * VE + e;
        if (c < a.cols) a.partial[(int64_t)blockIdx.x * a.cols + c] = dw[i * VE + e];
      }
  }
}

// dweight[c] = sum over the blocks' partial sums: 64 columns and 16 row
// streams a block
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* partial, int nblk, int cols, float* dw) {
  __shared__ float part[16][64];
  const int c = blockIdx.x * 64 + threadIdx.x % 64, r = threadIdx.x / 64;
  float s = 0.0f;
  if (c < cols)
    for (int b = r; b < nblk; b += 16) s += partial[(int64_t)b * cols + c];
  part[r][threadIdx.x % 64] = s;
  __syncthreads();
  if (r == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += part[i][threadIdx.x];
    dw[c] = s;
  }
}

// ------------------------------------------------------------ distillation --
// One pass: p = softmax(t / tau) over the row's teacher entries, q =
// softmax(z / tau) over all classes, loss = weight tau^2 sum p (log p - log q),
// dz = weight tau (q - p).  The row stays in registers between its maximum,
// its sum and its gradient (rows longer than 64 x 1024 are read twice).  The
// gradient is written as weight tau q first and the classes of the teacher's
// entries are then written again by the entries' threads; a class that several
// entries name is written by the first with all their p.
struct Teacher {  // LDS of one row
  int32_t idx[kDistillMaxK];
  float p[kDistillMaxK];
};

__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// Entry j is there: its index names a class (negative: left out) and its logit is not -inf.
__device__ __forceinline__ bool entry_there(int32_t i, float t) { return i >= 0 && !(t == -__builtin_inff()); }

template <typename T, int VE, int G, int EPT, bool STREAM>
__global__ __launch_bounds__(G > 256 ? G : 256) void distill_kernel(DistillArgs a) {
  constexpr int NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE;
  __shared__ float red[7][16];
  __shared__ Teacher teach[RPB];
  const int tid = threadIdx.x, t = tid % G;
  Teacher& te = teach[tid / G];
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
    const int64_t row0 = base + tid / G;
    const bool in = row0 < a.rows;      // every thread of the block stays for the barriers
    const int64_t row = in ? row0 : 0;
    const float weight = in ? (a.weight ? a.weight[row] : 1.0f) : 0.0f;
    // a row of weight 0 has loss 0 and gradient 0 whatever it holds: nothing of it is read
    const bool live = weight != 0.0f;
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz;
    const float inv_tau = 1.0f / a.tau;

    // the row's maximum, and the sum of exponentials
    float v[STREAM ? VE : EPT];
    float top = OpMax::zero, total = 0.0f;
    bool bad = false;
    if constexpr (!STREAM) {
  #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        if (live && c < a.classes) {
          load_vec<VE>(z + c, v + i * VE);
        } else {
  #pragma unroll
          for (int e = 0; e < VE; ++e) v[i * VE + e] = OpMax::zero;
        }
      }
      // the teacher's entries arrive while the row does
      for (int j = t; j < a.k; j += G) {
        te.idx[j] = live ? a.idx[row * a.k + j] : -1;
        te.p[j] = live ? a.teacher[row * a.k + j] : 0.0f;
      }
  #pragma unroll
      for (int e = 0; e < EPT; ++e) {
        top = fmaxf(top, v[e]);
        bad |= v[e] != v[e];
      }
      top = reduce_row<G, OpMax>(top, red[0], tid);
  #pragma unroll
      for (int i = 0; i < NV; ++i)
  #pragma unroll
        for (int e = 0; e < VE; ++e)
          if ((i * G + t) * VE + e < a.classes) total += fast_exp((v[i * VE + e] - top) * inv_tau);
    } else {
      for (int j = t; j < a.k; j += G) {
        te.idx[j] = live ? a.idx[row * a.k + j] : -1;
        te.p[j] = live ? a.teacher[row * a.k + j] : 0.0f;
      }
      if (live)
        for (int64_t c = (int64_t)t * VE; c < a.classes; c += (int64_t)G * VE) {
          load_vec<VE>(z + c, v);
          float m = top;
  #pragma unroll
          for (int e = 0; e < VE; ++e) {
            m = fmaxf(m, v[e]);
            bad |= v[e] != v[e];
          }
          if (m > top) {
            total *= fast_exp((top - m) * inv_tau);  // exp(-inf) = 0 the first time
            top = m;
          }
          if (top > OpMax::zero) {
  #pragma unroll
            for (int e = 0; e < VE; ++e) total += fast_exp((v[e] - top) * inv_tau);
          }
        }
      const float m = reduce_row<G, OpMax>(top, red[0], tid);
      total = top > OpMax::zero ? total * fast_exp((top - m) * inv_tau) : 0.0f;
      top = m;
    }
    if (bad) total = __builtin_nanf("");
    total = reduce_row<G, OpAdd>(total, red[1], tid);

    // the teacher's distribution (its entries were read by these same threads)
    float ttop = OpMax::zero;
    bool wrong = false;  // an index past the classes, or a NaN logit: the row's loss and gradient are NaN
    for (int j = t; j < a.k; j += G) {
      const int32_t i = te.idx[j];
      if (!entry_there(i, te.p[j])) {
        te.idx[j] = -1;
        continue;
      }
      wrong |= i >= a.classes || te.p[j] != te.p[j];
      if (i >= a.classes) te.idx[j] = -1;
      ttop = fmaxf(ttop, te.p[j]);
    }
    ttop = reduce_row<G, OpMax>(ttop, red[2], tid);
    float tsum = 0.0f;
    for (int j = t; j < a.k; j += G)
      if (te.idx[j] >= 0) tsum += fast_exp((te.p[j] - ttop) * inv_tau);
    tsum = reduce_row<G, OpAdd>(wrong ? __builtin_nanf("") : tsum, red[3], tid);
    const float log_tsum = logf(tsum), log_total = logf(total);
    float loss = 0.0f;
    for (int j = t; j < a.k; j += G) {
      const int32_t i = te.idx[j];
      if (i < 0) continue;
      const float lt = (te.p[j] - ttop) * inv_tau;
      const float p = fast_exp(lt) / tsum;
      const float lq = ((float)z[i] - top) * inv_tau - log_total;
      if (p != 0.0f) loss = fmaf(p, (lt - log_tsum) - lq, loss);
      te.p[j] = p;
    }
    loss = reduce_row<G, OpAdd>(loss, red[4], tid);
    const bool none = tsum == 0.0f;  // no entry is there: loss and gradient are 0
    if (in && t == 0) a.loss[row] = !live || none ? 0.0f : tsum != tsum ? tsum : weight * a.tau * a.tau * loss;

    if (!a.grad) {
      __syncthreads();  // the next row's entries and sums take the place of this one's
      continue;
    }
    T* g = static_cast<T*>(a.grad) + row * a.ldg;
    const float wt = weight * a.tau;
    const bool zero = !live || none;
    const float f = tsum != tsum ? tsum : wt / total;
    if constexpr (!STREAM) {
  #pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        if (in && c < a.classes) {
          float o[VE];
  #pragma unroll
          for (int e = 0; e < VE; ++e) o[e] = zero ? 0.0f : f * fast_exp((v[i * VE + e] - top) * inv_tau);
          store_vec<VE>(g + c, o);
        }
      }
    } else if (in) {
      for (int64_t c = (int64_t)t * VE; c < a.classes; c += (int64_t)G * VE) {
        float o[VE];
        if (!zero) load_vec<VE>(z + c, v);
  #pragma unroll
        for (int e = 0; e < VE; ++e) o[e] = zero ? 0.0f : f * fast_exp((v[e] - top) * inv_tau);
        store_vec<VE>(g + c, o);
      }
    }
    __syncthreads();  // the row's q are written, and every entry's p can be read
    for (int j = t; j < a.k && !zero; j += G) {
      const int32_t i = te.idx[j];
      if (i < 0) continue;
      float p = te.p[j];
      bool first = true;
      for (int o = 0; o < a.k; ++o)
        if (o != j && te.idx[o] == i) {
          if (o < j) first = false;
          p += te.p[o];
        }
      if (!first) continue;
      const float d = f * fast_exp(((float)z[i] - top) * inv_tau) - wt * p;
      g[i] = (T)d;
    }
    __syncthreads();  // before the next row's entries
  }
}

// blocks of a launch over rows, rpb of them a block (a launch is limited to
// 2^32 threads; a block goes on with the rows past the grid)
uint32_t row_blocks(int64_t rows, int rpb) {
  const int64_t n = (rows + rpb - 1) / rpb;
  return (uint32_t)(n < (1 << 20) ? n : 1 << 20);
}

template <typename T>
constexpr int kVec = 16 / sizeof(T);

template <typename T, int VE, int MODE>
hipError_t rows_t(const RowArgs& a, hipStream_t s) {
#define TABPACK_ROWS(G, EPT)                                                                        \
  if (a.cols <= G * EPT) {                                                                          \
    constexpr int RPB = G > 256 ? 1 : 256 / G;                                                      \
    hipLaunchKernelGGL((rows_kernel<T, VE, G, EPT, MODE>), dim3(row_blocks(a.rows, RPB)),       \
                       dim3(G > 256 ? G : 256), 0, s, a);                                           \
    return hipGetLastError();                                                                       \
  }
  TABPACK_ROWS(64, 8)
  TABPACK_ROWS(64, 16)
  TABPACK_ROWS(64, 32)
  TABPACK_ROWS(256, 16)
  TABPACK_ROWS(256, 32)
  TABPACK_ROWS(1024, 16)
  TABPACK_ROWS(1024, 32)
#undef TABPACK_ROWS
  return hipErrorInvalidValue;
}
template <typename T, int MODE>
hipError_t rows_m(const RowArgs& a, hipStream_t s) {
  return a.vec ? rows_t<T, kVec<T>, MODE>(a, s) : rows_t<T, 1, MODE>(a, s);
}
template <typename T>
hipError_t rows_p(RowMode mode, const RowArgs& a, hipStream_t s) {
  switch (mode) {
    case ROW_NORM: return rows_m<T, ROW_NORM>(a, s);
    case ROW_NORM_Q8: return rows_m<T, ROW_NORM_Q8>(a, s);
    default: return rows_m<T, ROW_Q8>(a, s);
  }
}

template <typename T, int VE>
hipError_t norm_bwd_t(const NormBwdArgs& a, hipStream_t s) {
  const int nblk = norm_bwd_blocks(a.rows, a.cols);
#define TABPACK_NORM_BWD(G, EPT)                                                                             \
  if (a.cols <= G * EPT) {                                                                                   \
    hipLaunchKernelGGL((norm_bwd_kernel<T, VE, G, EPT>), dim3(nblk), dim3(G > 256 ? G : 256), 0, s, a);       \
    hipLaunchKernelGGL(norm_dw_kernel, dim3((a.cols + 63) / 64), dim3(1024), 0, s, a.partial, nblk, a.cols,   \
                       a.dweight);                                                                           \
    return hipGetLastError();                                                                                \
  }
  TABPACK_NORM_BWD(64, 8)
  TABPACK_NORM_BWD(64, 16)
  TABPACK_NORM_BWD(64, 32)
  TABPACK_NORM_BWD(256, 16)
  TABPACK_NORM_BWD(256, 32)
  TABPACK_NORM_BWD(1024, 16)
  TABPACK_NORM_BWD(1024, 32)
#undef TABPACK_NORM_BWD
  return hipErrorInvalidValue;
}

template <typename T, int VE>
hipError_t distill_t(const DistillArgs& a, hipStream_t s) {
#define TABPACK_DISTILL(G, EPT, STREAM)                                                                        \
  if (STREAM || a.classes <= G * EPT) {                                                                        \
    constexpr int RPB = G > 256 ? 1 : 256 / G;                                                                 \
    hipLaunchKernelGGL((distill_kernel<T, VE, G, EPT, STREAM>), dim3(row_blocks(a.rows, RPB)),     \
                       dim3(G > 256 ? G : 256), 0, s, a);                                                      \
    return hipGetLastError();                                                                                  \
  }
  TABPACK_DISTILL(16, 8, false)
  TABPACK_DISTILL(64, 16, false)
  TABPACK_DISTILL(256, 16, false)
  TABPACK_DISTILL(1024, 16, false)
  TABPACK_DISTILL(1024, 32, false)
  TABPACK_DISTILL(1024, 64, false)
  TABPACK_DISTILL(1024, VE, true)
#undef TABPACK_DISTILL
}

}  // namespace

hipError_t launch_rows(int prec, RowMode mode, const RowArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? rows_p<__bf16>(mode, a, s) : rows_p<float>(mode, a, s);
}

// rows that share a block's weight sums: enough blocks to fill the chip four
// times over, few enough that adding up their sums is a small part
int norm_bwd_blocks(int64_t rows, int32_t cols) {
  const int64_t per = cols <= 2048 ? 4 : 1;  // rows a block takes at a time
  const int64_t want = (rows + per - 1) / per;
  return (int)(want < 1024 ? (want > 0 ? want : 1) : 1024);
}

hipError_t launch_norm_bwd(int prec, const NormBwdArgs& a, hipStream_t s) {
  if (prec == PACK_PREC_BF16) return a.vec ? norm_bwd_t<__bf16, 8>(a, s) : norm_bwd_t<__bf16, 1>(a, s);
  return a.vec ? norm_bwd_t<float, 4>(a, s) : norm_bwd_t<float, 1>(a, s);
}

hipError_t launch_distill(int prec, const DistillArgs& a, hipStream_t s) {
  if (prec == PACK_PREC_BF16) return a.vec ? distill_t<__bf16, 8>(a, s) : distill_t<__bf16, 1>(a, s);
  return a.vec ? distill_t<float, 4>(a, s) : distill_t<float, 1>(a, s);
}

}  // namespace tabpack
