// Row kernels of the student network on gfx950: the root-mean-square norm with
// the residual's addition (forward, 8-bit output, backward), row quantisation,
// and distillation from a teacher's top logits.
//
// Each does a few operations a byte, so the bytes of one read and one write
// bound it.  A row is read once into the registers of the G threads that own
// it (4 to 1024, EPT elements each, by the row's length), reduced there, and
// written from there.  Thread t of a row owns the vectors t, t + G, t + 2G, ...
// of VE elements (16 bytes), so a wave's accesses are contiguous.  Vectors are
// accessed at any alignment of the element (the global memory path splits what
// crosses a line); the one that the row's end cuts is accessed by elements.
// Sums are held in fp32 and added in a fixed order.
//
// Measured on tensors larger than the caches, against 5.1 TB/s of a device copy:
// norm with residual 65,536 x 1024 bf16 93 us (5.8 TB/s of reads and writes),
// with 8-bit output 88 us, its backward with both gradients 106 us (5.1 TB/s),
// quantising 35 us (5.8 TB/s); 500,000 x 64 bf16 norm 53 us (4 and 16 threads a
// row: a wave a row takes 181); distillation 4096 x 32,000 bf16 with 32 entries
// a row 120 us (4.4 TB/s).  Odd lengths (4095) cost up to 1.3 times the time in
// bf16, whose stores then share their lines; rows of 32,768 in the backward pass
// 4 times, whose column sums no longer fit the registers.
#include "ops_internal.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
// the same at any alignment
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef f32x4 f32x4_any __attribute__((aligned(1)));

template <typename T>
constexpr int kVec = 16 / sizeof(T);

// A vector as it lies in memory, and its elements as floats
template <typename T>
struct Vec {
  u32x4 raw;
  // the first n elements at p (all kVec where n says so or more), the others `fill`
  __device__ __forceinline__ void load(const T* p, int n, float fill = 0.0f) {
    if (n >= kVec<T>) {
      raw = *reinterpret_cast<const u32x4_any*>(p);
    } else {
      T e[kVec<T>];
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) e[i] = i < n ? p[i] : (T)fill;
      __builtin_memcpy(&raw, e, 16);
    }
  }
  __device__ __forceinline__ void get(float* v) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xffff0000u);
      }
    } else {
      const f32x4 f = __builtin_bit_cast(f32x4, raw);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = f[i];
    }
  }
};
// the first n (at most kVec) of kVec values
__device__ __forceinline__ void store_vec(__bf16* p, const float* v, int n) {
  bf16x8 o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
  if (n >= 8) {
    *reinterpret_cast<u32x4_any*>(p) = __builtin_bit_cast(u32x4, o);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = o[i];
  }
}
__device__ __forceinline__ void store_vec(float* p, const float* v, int n) {
  if (n >= 4) {
    *reinterpret_cast<f32x4_any*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}
// N of the n weights at p; those past the end are 0
template <int N>
__device__ __forceinline__ void load_weight(const float* p, float* w, int n) {
  if (n >= N) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const f32x4 f = *reinterpret_cast<const f32x4_any*>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = f[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = i < n ? p[i] : 0.0f;
  }
}
// N codes (whole numbers in [-127, 127]), the first n
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const float* v, int n) {
  if (n >= N) {
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i] |= ((uint32_t)(int32_t)v[4 * i + j] & 0xffu) << (8 * j);
    }
    if constexpr (N == 8)
      *reinterpret_cast<u32x2_any*>(p) = u32x2{w[0], w[1]};
    else
      *reinterpret_cast<u32_any*>(p) = w[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = (int8_t)(int32_t)v[i];
  }
}

struct OpAdd {
  __device__ static float op(float a, float b) { return a + b; }
};
// Largest of values that are not negative; NaN counts as larger than infinity
// (the order of their bits), so it is not lost.
struct OpMaxMag {
  __device__ static float op(float a, float b) {
    return __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)));
  }
};
struct OpMax {
  __device__ static float op(float a, float b) { return fmaxf(a, b); }
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
// holds an infinity or NaN gets codes 0 and scale NaN.  Where the squares
// overflow (values past 1.8e19) the row goes on 2^-80 times smaller, which
// changes neither y nor the codes.
template <typename T, int G, int EPT, int MODE>
__global__ __launch_bounds__(G > 256 ? G : 256) void rows_kernel(RowArgs a) {
  constexpr int VE = kVec<T>, NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE;
  __shared__ float red[2][3][16];
  const int tid = threadIdx.x, t = tid % G;
  static_assert(G <= 64 || RPB == 1, "a row's barriers are the block's");
  int turn = 0;  // rows take turns with two sets of LDS words: a row's barriers lie between their uses
  for (int64_t row = (int64_t)blockIdx.x * RPB + tid / G; row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const bool add = MODE != ROW_Q8 && a.residual;
    const T* r = add ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
    Vec<T> xs[NV], rs[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      xs[i].load(x + c, a.cols - c);
      if (add) rs[i].load(r + c, a.cols - c);
    }
    float v[EPT];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      xs[i].get(v + i * VE);
      if (add) {
        float u[VE];
        rs[i].get(u);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[i * VE + e] += u[e];
      }
    }
    float rho = 1.0f;
    if constexpr (MODE != ROW_Q8) {
      if (a.sum) {
        T* s = static_cast<T*>(a.sum) + row * a.lds;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VE;
          store_vec(s + c, v + i * VE, a.cols - c);
        }
      }
      float sq = 0.0f;
#pragma unroll
      for (int e = 0; e < EPT; ++e) sq = fmaf(v[e], v[e], sq);
      sq = reduce_row<G, OpAdd>(sq, red[turn][0], tid);
      rho = 1.0f / sqrtf(sq / (float)a.cols + a.eps);
      float rstd = rho;
      if (!(sq < __builtin_inff())) {  // (the same for all threads of the row)
        constexpr float kDown = 0x1p-80f;
        float down = 0.0f;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
          v[e] *= kDown;
          down = fmaf(v[e], v[e], down);
        }
        down = reduce_row<G, OpAdd>(down, red[turn][2], tid);
        rho = 1.0f / sqrtf(down / (float)a.cols + a.eps * kDown * kDown);
        rstd = rho * kDown;
      }
      if (a.rstd && t == 0) a.rstd[row] = rstd;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        float w[VE];
        load_weight<VE>(a.weight + c, w, a.cols - c);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          float& y = v[i * VE + e];
          y = MODE == ROW_NORM ? y * rho * w[e] : y * w[e];
        }
      }
    }
    if constexpr (MODE == ROW_NORM) {
      T* o = static_cast<T*>(a.out) + row * a.ldo;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        store_vec(o + c, v + i * VE, a.cols - c);
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
        float k[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) k[e] = finite ? rintf(v[i * VE + e] * f) : 0.0f;
        store_codes<VE>(q + c, k, a.cols - c);
      }
    }
  }
}

// --------------------------------------------------------- norm, backward --
// With g = w dy, rho as saved, n = v rho and D = cols:
//   dx = rho (g - n / D sum_c g n) + dsum,   dweight = sum_rows dy n.
// (The products are with n, of order 1 whatever the row's magnitude: those with v
// and rho^2 leave fp32's range where v is large.)
// A block walks over rows (gridDim apart) and keeps the columns' weight sums
// in registers; its sums go to one row of `partial`, which a second kernel
// adds up in order: no atomics, so the result does not change between runs.
template <typename T, int G, int EPT>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int VE = kVec<T>, NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE;
  __shared__ float red[2][16];
  __shared__ float cols[RPB > 1 ? G * EPT : 1];
  const int tid = threadIdx.x, t = tid % G, rg = tid / G;
  float dw[EPT];
#pragma unroll
  for (int e = 0; e < EPT; ++e) dw[e] = 0.0f;
  int turn = 0;  // (as in rows_kernel)
  for (int64_t row = (int64_t)blockIdx.x * RPB + rg; row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
    const T* s = static_cast<const T*>(a.sum) + row * a.lds;
    const T* dy = static_cast<const T*>(a.dy) + row * a.ldy;
    const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.ldd : nullptr;
    Vec<T> vs[NV], gs[NV], os[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      vs[i].load(s + c, a.cols - c);
      gs[i].load(dy + c, a.cols - c);
      if (ds)
        os[i].load(ds + c, a.cols - c);
      else
        os[i].raw = u32x4{0, 0, 0, 0};
    }
    const float rho = a.rstd[row];
    // bf16 keeps n and g as floats; fp32 keeps n in v's place and forms g, the weight
    // read again from the cache, a second time (16,384 x 4096: bf16 93 us against 99 the other
    // way, fp32 156 against 183)
    constexpr bool KEEP = sizeof(T) == 2;
    float kv[KEEP ? EPT : 1], kg[KEEP ? EPT : 1], dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      float w[VE], v[VE], g[VE];
      load_weight<VE>(a.weight + c, w, a.cols - c);
      vs[i].get(v);
      gs[i].get(g);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        v[e] *= rho;
        dw[i * VE + e] = fmaf(g[e], v[e], dw[i * VE + e]);
        g[e] *= w[e];
        dot = fmaf(g[e], v[e], dot);
        if constexpr (KEEP) kv[i * VE + e] = v[e], kg[i * VE + e] = g[e];
      }
      if constexpr (!KEEP) vs[i].raw = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    }
    dot = reduce_row<G, OpAdd>(dot, red[turn], tid);
    const float c1 = dot / (float)a.cols;
    T* dx = static_cast<T*>(a.dx) + row * a.ldx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      float v[VE], g[VE], o[VE];
      if constexpr (KEEP) {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = kv[i * VE + e], g[e] = kg[i * VE + e];
      } else {
        float w[VE];
        load_weight<VE>(a.weight + c, w, a.cols - c);
        vs[i].get(v);
        gs[i].get(g);
#pragma unroll
        for (int e = 0; e < VE; ++e) g[e] *= w[e];
      }
      os[i].get(o);
#pragma unroll
      for (int e = 0; e < VE; ++e) o[e] = fmaf(rho, g[e] - v[e] * c1, o[e]);
      store_vec(dx + c, o, a.cols - c);
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

// dweight[c] = sum over the blocks' partial sums: 16 columns and 64 row streams
// a block
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* partial, int nblk, int cols, float* dw) {
  __shared__ float part[64][17];
  const int i = threadIdx.x % 16, c = blockIdx.x * 16 + i, r = threadIdx.x / 16;
  float s = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int b = r; b < nblk; b += 64) s += partial[(int64_t)b * cols + c];
  }
  part[r][i] = s;
  __syncthreads();
  if (r == 0 && c < cols) {
    for (int q = 1; q < 64; ++q) s += part[q][i];
    dw[c] = s;
  }
}

// ------------------------------------------------------------ distillation --
// One pass: p = softmax(t / tau) over the row's teacher entries, q =
// softmax(z / tau) over all classes, loss = weight tau^2 sum p (log p - log q),
// dz = weight tau (q - p).  The row stays in registers as it was read between
// its maximum, its sum and its gradient (rows longer than 64 x 1024 are read
// twice, the first time with a running maximum and sum).  The row's first
// threads take the teacher's entries meanwhile.  The gradient is written as
// weight tau q first and the classes of the teacher's entries are then written
// again by their threads; a class that several entries name is written by the
// first of them with all their p.  512 threads hold up to 32,768 classes, so two
// rows share a CU and one's reads run beside the other's exponentials (1024
// threads with one row a CU: 233 us for the case above).
struct Teacher {  // LDS of one row: k entries of each, and the sum
  int32_t* idx;  // class, or -1
  float* p;      // logit, then p
  float* z;      // the student's logit of the class
  float* sum;    // of exp((t - largest t) / tau): 0 without entries, NaN for a row that is wrong
  __device__ Teacher(char* lds, int k)
      : idx(reinterpret_cast<int32_t*>(lds)), p(reinterpret_cast<float*>(lds) + k), z(p + k), sum(z + k) {}
};
int teacher_bytes(int k) { return (3 * k + 1) * 4; }

__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

template <typename T, int G, int EPT, bool STREAM>
__global__ __launch_bounds__(G > 256 ? G : 256) void distill_kernel(DistillArgs a) {
  constexpr int VE = kVec<T>, NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE, W = G < 64 ? G : 64;
  __shared__ float red[2][16];
  extern __shared__ char teach[];
  const int tid = threadIdx.x, t = tid % G;
  const Teacher te(teach + (tid / G) * ((3 * a.k + 1) * 4), a.k);
  const float inv_tau = 1.0f / a.tau;
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
    const bool in = base + tid / G < a.rows;  // every thread of the block stays for the barriers
    const int64_t row = in ? base + tid / G : 0;
    const float weight = in ? (a.weight ? a.weight[row] : 1.0f) : 0.0f;
    // a row of weight 0 has loss 0 and gradient 0 whatever it holds: nothing of it is read
    const bool live = weight != 0.0f;
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz;
    constexpr float kNone = -__builtin_inff();

    Vec<T> zs[NV];
    if constexpr (!STREAM) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        zs[i].load(z + c, live ? a.classes - c : 0, kNone);
      }
    }
    if (t < W) {
      // an entry is there if its index is not negative and its logit not -inf
      float ttop = kNone;
      bool wrong = false;  // an index past the classes or a NaN logit
      for (int j = t; j < a.k; j += W) {
        const int32_t i = live ? a.idx[row * a.k + j] : -1;
        const float l = live ? a.teacher[row * a.k + j] : 0.0f;
        const bool there = i >= 0 && l != kNone, known = there && i < a.classes;
        wrong |= there && (!known || l != l);
        te.idx[j] = known ? i : -1;
        te.p[j] = l;
        te.z[j] = known ? (float)z[i] : 0.0f;
        if (known) ttop = fmaxf(ttop, l);
      }
#pragma unroll
      for (int m = W / 2; m >= 1; m >>= 1) ttop = fmaxf(ttop, __shfl_xor(ttop, m, 64));
      float tsum = 0.0f;
      for (int j = t; j < a.k; j += W)
        if (te.idx[j] >= 0) {
          te.p[j] = (te.p[j] - ttop) * inv_tau;
          tsum += fast_exp(te.p[j]);
        }
      if (wrong) tsum = __builtin_nanf("");
#pragma unroll
      for (int m = W / 2; m >= 1; m >>= 1) tsum += __shfl_xor(tsum, m, 64);
      if (t == 0) *te.sum = tsum;  // (the others read it after the next barrier, or are of this wave)
    }

    // the row's maximum, and the sum of exponentials (a NaN makes the sum NaN)
    float top = kNone, total = 0.0f;
    if constexpr (!STREAM) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float v[VE];
        zs[i].get(v);
#pragma unroll
        for (int e = 0; e < VE; ++e) top = fmaxf(top, v[e]);
      }
      top = reduce_row<G, OpMax>(top, red[0], tid);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float v[VE];
        zs[i].get(v);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          // (places past the classes hold -inf: exp gives 0 unless the row has nothing above -inf)
          const float x = fast_exp((v[e] - top) * inv_tau);
          total += top > kNone || (i * G + t) * VE + e < a.classes ? x : 0.0f;
        }
      }
    } else {
      bool bad = false;
      if (live)
        for (int64_t c = (int64_t)t * VE; c < a.classes; c += (int64_t)G * VE) {
          Vec<T> y;
          float v[VE], m = top;
          y.load(z + c, (int)min((int64_t)VE, a.classes - c), kNone);
          y.get(v);
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            m = fmaxf(m, v[e]);
            bad |= v[e] != v[e];
          }
          if (m > top) {
            total *= fast_exp((top - m) * inv_tau);  // exp(-inf) = 0 the first time
            top = m;
          }
          if (top > kNone) {
#pragma unroll
            for (int e = 0; e < VE; ++e) total += fast_exp((v[e] - top) * inv_tau);
          }
        }
      const float m = reduce_row<G, OpMax>(top, red[0], tid);
      total = bad || m == kNone ? __builtin_nanf("") : top > kNone ? total * fast_exp((top - m) * inv_tau) : 0.0f;
      top = m;
    }
    total = reduce_row<G, OpAdd>(total, red[1], tid);
    if constexpr (G <= 64) {  // (wider rows had a block barrier since lane 0 wrote the entries' sum)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }

    const float tsum = *te.sum;
    const bool zero = !live || tsum == 0.0f;  // nothing of the row counts
    const float wt = weight * a.tau, f = tsum != tsum ? tsum : wt / total;
    if (t < W) {
      const float log_tsum = logf(tsum), log_total = logf(total);
      float loss = 0.0f;
      for (int j = t; j < a.k; j += W) {
        if (te.idx[j] < 0) continue;
        const float lt = te.p[j], p = fast_exp(lt) / tsum;
        te.p[j] = p;
        if (p != 0.0f) loss = fmaf(p, (lt - log_tsum) - ((te.z[j] - top) * inv_tau - log_total), loss);
      }
#pragma unroll
      for (int m = W / 2; m >= 1; m >>= 1) loss += __shfl_xor(loss, m, 64);
      if (in && t == 0)
        a.loss[row] = zero ? 0.0f : tsum != tsum || total != total ? __builtin_nanf("") : wt * a.tau * loss;
    }
    if (a.grad) {
      T* g = static_cast<T*>(a.grad) + row * a.ldg;
      if constexpr (!STREAM) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VE;
          float o[VE];
          zs[i].get(o);
#pragma unroll
          for (int e = 0; e < VE; ++e) o[e] = zero ? 0.0f : f * fast_exp((o[e] - top) * inv_tau);
          store_vec(g + c, o, in ? a.classes - c : 0);
        }
      } else if (in) {
        for (int64_t c = (int64_t)t * VE; c < a.classes; c += (int64_t)G * VE) {
          const int n = (int)min((int64_t)VE, a.classes - c);
          Vec<T> y;
          float o[VE];
          y.load(z + c, zero ? 0 : n, kNone);
          y.get(o);
#pragma unroll
          for (int e = 0; e < VE; ++e) o[e] = zero ? 0.0f : f * fast_exp((o[e] - top) * inv_tau);
          store_vec(g + c, o, n);
        }
      }
      __syncthreads();  // the row's q are written, and every entry's p can be read
      for (int j = t; t < W && j < a.k && !zero; j += W) {
        const int32_t i = te.idx[j];
        if (i < 0) continue;
        float p = te.p[j];
        bool first = true;
        for (int o = 0; o < a.k; ++o)
          if (o != j && te.idx[o] == i) {
            if (o < j) first = false;
            p += te.p[o];
          }
        if (first) g[i] = (T)(f * fast_exp((te.z[j] - top) * inv_tau) - wt * p);
      }
    }
    if (base + (int64_t)gridDim.x * RPB < a.rows) __syncthreads();  // before the next row's entries and sums
  }
}

// blocks of a launch over rows, rpb of them a block (a launch is limited to
// 2^32 threads; a block goes on with the rows past the grid)
uint32_t row_blocks(int64_t rows, int rpb) {
  const int64_t n = (rows + rpb - 1) / rpb;
  return (uint32_t)(n < (1 << 20) ? n : 1 << 20);
}

template <typename T, int MODE>
hipError_t rows_t(const RowArgs& a, hipStream_t s) {
#define TABPACK_ROWS(G, EPT)                                                                        \
  if (a.cols <= G * EPT) {                                                                          \
    constexpr int RPB = G > 256 ? 1 : 256 / G;                                                      \
    hipLaunchKernelGGL((rows_kernel<T, G, EPT, MODE>), dim3(row_blocks(a.rows, RPB)),       \
                       dim3(G > 256 ? G : 256), 0, s, a);                                           \
    return hipGetLastError();                                                                       \
  }
  TABPACK_ROWS(4, 8)
  TABPACK_ROWS(16, 8)
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
template <typename T>
hipError_t rows_p(RowMode mode, const RowArgs& a, hipStream_t s) {
  switch (mode) {
    case ROW_NORM: return rows_t<T, ROW_NORM>(a, s);
    case ROW_NORM_Q8: return rows_t<T, ROW_NORM_Q8>(a, s);
    default: return rows_t<T, ROW_Q8>(a, s);
  }
}

template <typename T>
hipError_t norm_bwd_t(const NormBwdArgs& a, hipStream_t s) {
  const int nblk = norm_bwd_blocks(a.rows, a.cols);
#define TABPACK_NORM_BWD(G, EPT)                                                                             \
  if (a.cols <= G * EPT) {                                                                                   \
    hipLaunchKernelGGL((norm_bwd_kernel<T, G, EPT>), dim3(nblk), dim3(G > 256 ? G : 256), 0, s, a);       \
    hipLaunchKernelGGL(norm_dw_kernel, dim3((a.cols + 15) / 16), dim3(1024), 0, s, a.partial, nblk, a.cols,   \
                       a.dweight);                                                                           \
    return hipGetLastError();                                                                                \
  }
  TABPACK_NORM_BWD(4, 8)
  TABPACK_NORM_BWD(16, 8)
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

template <typename T>
hipError_t distill_t(const DistillArgs& a, hipStream_t s) {
#define TABPACK_DISTILL(G, EPT, STREAM)                                                                        \
  if (STREAM || a.classes <= G * EPT) {                                                                        \
    constexpr int RPB = G > 256 ? 1 : 256 / G;                                                                 \
    hipLaunchKernelGGL((distill_kernel<T, G, EPT, STREAM>), dim3(row_blocks(a.rows, RPB)),     \
                       dim3(G > 256 ? G : 256), RPB * teacher_bytes(a.k), s, a);                               \
    return hipGetLastError();                                                                                  \
  }
  if (a.k <= 32) {  // (64 rows' entries in LDS)
    TABPACK_DISTILL(4, 8, false)
  }
  TABPACK_DISTILL(16, 8, false)
  TABPACK_DISTILL(64, 16, false)
  TABPACK_DISTILL(256, 16, false)
  TABPACK_DISTILL(256, 32, false)
  TABPACK_DISTILL(512, 32, false)
  TABPACK_DISTILL(512, 64, false)
  TABPACK_DISTILL(1024, 64, false)
  TABPACK_DISTILL(1024, kVec<T>, true)
#undef TABPACK_DISTILL
}

}  // namespace

hipError_t launch_rows(int prec, RowMode mode, const RowArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? rows_p<__bf16>(mode, a, s) : rows_p<float>(mode, a, s);
}

// rows that share a block's weight sums: enough blocks to fill the chip four
// times over, few enough that adding up their sums is a small part
int norm_bwd_blocks(int64_t rows, int32_t cols) {
  const int64_t per = cols <= 32 ? 64 : cols <= 128 ? 16 : cols <= 2048 ? 4 : 1;  // rows a block takes at a time
  const int64_t want = (rows + per - 1) / per;
  return (int)(want < 1024 ? (want > 0 ? want : 1) : 1024);
}

hipError_t launch_norm_bwd(int prec, const NormBwdArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? norm_bwd_t<__bf16>(a, s) : norm_bwd_t<float>(a, s);
}

hipError_t launch_distill(int prec, const DistillArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? distill_t<__bf16>(a, s) : distill_t<float>(a, s);
}

}  // namespace tabpack
