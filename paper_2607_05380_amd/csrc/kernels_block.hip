// Matrix products of the student network on gfx950: the gated feed-forward
// block (forward and backward, bf16 and fp32) and the 8-bit product with a
// scale per row and per output, plain or gated.
//
// All of them are C[m, n] = sum_k A(m, k) B(n, k) with an epilogue per element
// (MmEpi).  Operands are depth-contiguous or rows-contiguous, so that the
// backward products read the same matrices as the forward ones and nothing is
// transposed in memory:
//   [g | u] = x Wgu^T    A = x  (K),   B = Wgu (K), epilogue h = act(g) u
//   y = h Wd^T           A = h  (K),   B = Wd  (K)
//   dh = dy Wd           A = dy (K),   B = Wd  (R), epilogue [dg | du]
//   dx = [dg | du] Wgu   A = dgu (K),  B = Wgu (R)
//   dWgu = [dg | du]^T x A = dgu (R),  B = x   (R)
//   dWd = dy^T h         A = dy (R),   B = h   (R)
// A gated tile takes as many gate rows of B as up rows, laid out so that a
// lane's accumulators hold both values of an output: the activation and the
// product cost no pass over memory.
//
// A K step is 128 bytes of depth (64 bf16, 128 int8, 32 fp32).  Tiles (times:
// bf16 products of M x N x K):
//   small  128 x 128, 4 waves of 64 x 64, two steps in LDS (64 KB), two
//          workgroups per CU.  Operands go straight to LDS; those whose rows do
//          not start at 16 bytes or end inside a 16-byte vector, where copying
//          them first takes longer (see copies()), pass through registers, two
//          steps ahead.  2048 x 4096 x 1024 22 us
//          (0.8 PFLOP/s; huge 30, mini 31), through registers 31.  fp32: 4096 x
//          1024 gated x 512 70 us (123 TFLOP/s; a library product of 8192 a
//          side 153), through registers 78.
//   huge   256 x 256, 8 waves of 128 x 64, 160 KB of LDS, one workgroup per CU
//          (see huge_tile).  16,384 x 1024 x 4096 107 us (1.29 PFLOP/s; small
//          128), where a large library product reaches 1.42.
//   mini   64 x 64, 4 waves of 32 x 32, four steps in LDS (64 KB); for products
//          whose larger tiles would leave CUs idle.  2048 x 1024 x 1024 10 us
//          (small 13.5, huge 24).
//   thin   up to 16 rows of A, 16 columns, no LDS for operands: each weight
//          byte is read once (see thin_kernel).
// What bounds the large tiles is power: with random operands the MFMAs alone,
// without loads or LDS reads, take 0.82 of the time of the whole loop, and with
// zeros the loop is 1.4 times faster.
// MFMAs: v_mfma_f32_32x32x16_bf16, v_mfma_i32_32x32x32_i8,
// v_mfma_f32_32x32x2_f32, with B as the first operand, so that a lane holds 4
// consecutive columns of one row of C.  Accumulators are fp32 or int32, added
// in a fixed order; a depth split over workgroups is joined in a fixed order
// by a second kernel.  What is rounded to bf16 between two products (h, dg and du)
// is rounded once, from fp32, since the next product's instructions take bf16; g and
// u are saved in fp32.  So a gradient in bf16 has sqrt(2) times the error of its own
// rounding.  With g and u rounded as well it had 1.8 times, in a training step of
// 16,384 tokens of 1024, hidden 4096, that took 1206 us instead of 1321 (2048
// tokens 216, 229): the bytes of the two gate epilogues bound the difference.
#include <algorithm>
#include <cmath>

#include "gemm_tiles.h"
#include "ops_internal.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int kStep = 128;           // bytes of depth per K step
constexpr int kRegion = 128 * kStep; // one operand region of a K step in LDS

template <typename T>
struct Ty;
template <>
struct Ty<__bf16> {
  typedef float acc_t;
  typedef f32x16 acc16;
  static constexpr int VE = 8;
};
template <>
struct Ty<float> {
  typedef float acc_t;
  typedef f32x16 acc16;
  static constexpr int VE = 4;
};
template <>
struct Ty<int8_t> {
  typedef int32_t acc_t;
  typedef i32x16 acc16;
  static constexpr int VE = 16;
};

constexpr bool is_gate(int epi) { return epi == MM_GATE || epi == MM_Q8_GATE; }
constexpr bool is_q8(int epi) { return epi == MM_Q8 || epi == MM_Q8_GATE; }

// -------------------------------------------------------------- activations --
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * -1.4426950408889634f); }
// the logistic function, with the hardware's reciprocal (1 ulp; a division
// costs ten instructions more)
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_neg(x)); }
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
// The normal distribution function at g, with e = exp(-g^2 / 2).  The tail beyond
// x = |g| is e t P(t) with t = 1 / (1 + 0.31 x): its quotient by e falls like 1 / x
// and is smooth in t.  P, of degree 7, was fitted in the largest relative error over
// 0 <= x <= 14 (1.6e-7; evaluated in fp32 4.5e-7; e is 0 further out), so the
// negative side keeps its leading digits, where 1 + erf would be a difference of
// large values.  No branches.
__device__ __forceinline__ float normal_cdf(float g, float e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.31f, 1.0f));
  float p = fmaf(t, 0.0358418226f, -0.141604945f);
  p = fmaf(t, p, 0.155068398f);
  p = fmaf(t, p, -0.0149038201f);
  p = fmaf(t, p, 0.110110328f);
  p = fmaf(t, p, 0.107771039f);
  p = fmaf(t, p, 0.124060348f);
  p = fmaf(t, p, 0.123656906f);
  const float tail = t * p * e;
  return g < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float exp_half_square(float g) {
  return __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f);
}

// c <- act(c) u, 8 values (the choice of the activation outside their loop)
__device__ __forceinline__ void gate8(int act, float* c, const float* u) {
  if (act == PACK_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = c[i] * logistic(c[i]) * u[i];
  } else if (act == PACK_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = c[i] * normal_cdf(c[i], exp_half_square(c[i])) * u[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = (c[i] > 0.0f ? c[i] : c[i] == c[i] ? 0.0f : c[i]) * u[i];
  }
}
// g <- d u act'(g) and u <- d act(g): the gradients of gate and up from d = dh
__device__ __forceinline__ void gate8_grad(int act, const float* d, float* g, float* u) {
  if (act == PACK_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = logistic(g[i]), v = g[i] * p;
      g[i] = d[i] * u[i] * (p + v * (1.0f - p));
      u[i] = d[i] * v;
    }
  } else if (act == PACK_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e = exp_half_square(g[i]), c = normal_cdf(g[i], e), v = g[i] * c;
      g[i] = d[i] * u[i] * fmaf(g[i] * kInvSqrt2Pi, e, c);
      u[i] = d[i] * v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = g[i] > 0.0f ? g[i] : g[i] == g[i] ? 0.0f : g[i];
      g[i] = d[i] * u[i] * (g[i] > 0.0f ? 1.0f : 0.0f);
      u[i] = d[i] * v;
    }
  }
}

// ---------------------------------------------------------------- epilogues --
// the same at any alignment (the global memory path splits what crosses a line)
typedef u32x4 u32x4_any __attribute__((aligned(1)));

// 8 consecutive elements as they lie in memory
template <typename T>
struct Raw8 {
  u32x4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = *reinterpret_cast<const u32x4_any*>(p + i * (16 / sizeof(T)));
  }
  // n (1 to 8) elements exist: the others repeat the last one (loads without a
  // branch, so none waits for another)
  __device__ __forceinline__ void load(const T* p, int n) {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = p[min(i, n - 1)];
    __builtin_memcpy(v, e, sizeof v);
  }
  template <bool PART>
  __device__ __forceinline__ void load_some(const T* p, int n) {
    if constexpr (PART)
      load(p, n);
    else
      load(p);
  }
  __device__ __forceinline__ void get(float* f) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __builtin_bit_cast(float, v[0][i] << 16);
        f[2 * i + 1] = __builtin_bit_cast(float, v[0][i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 x = __builtin_bit_cast(f32x4, v[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[4 * i + j] = x[j];
      }
    }
  }
};
__device__ __forceinline__ void store8(__bf16* p, const float* v) {
  bf16x8 o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
  *reinterpret_cast<u32x4_any*>(p) = __builtin_bit_cast(u32x4, o);
}
__device__ __forceinline__ void store8(float* p, const float* v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 x{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
    *reinterpret_cast<u32x4_any*>(p + 4 * i) = __builtin_bit_cast(u32x4, x);
  }
}

// 8 values, or the first n of them
template <bool PART, typename T>
__device__ __forceinline__ void store_some(T* p, const float* v, int n) {
  if constexpr (!PART) {
    store8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

// What an epilogue reads besides the sums, for 8 columns (PART: for the first
// cnt of them): per column (8-bit
// products), and per row and column.
template <bool PART>
struct Q8Cols {
  Raw8<float> scale, bias;
  __device__ __forceinline__ void load(const MmArgs& a, int n, int cnt) {
    scale.template load_some<PART>(a.col_scale + n, cnt);
    if (a.bias) bias.template load_some<PART>(a.bias + n, cnt);
  }
  // sums in int32 -> values
  __device__ __forceinline__ void apply(const MmArgs& a, float* c, float row_scale) const {
    float s[8];
    scale.get(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = (float)__builtin_bit_cast(int32_t, c[i]) * (row_scale * s[i]);
    if (a.bias) {
      float b[8];
      bias.get(b);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] += b[i];
    }
  }
};
template <int EPI, typename T, bool PART>
struct Cols {
  Q8Cols<PART> gate, up;
  __device__ __forceinline__ void load(const MmArgs& a, int n, int cnt) {
    if constexpr (is_q8(EPI)) gate.load(a, n, cnt);
    if constexpr (EPI == MM_Q8_GATE) up.load(a, a.N + n, cnt);
  }
};
template <int EPI, typename T, bool PART>
struct Extra {
  Raw8<std::conditional_t<EPI == MM_GATE_BWD, float, T>> g, u;
  float row_scale;
  __device__ __forceinline__ void load(const MmArgs& a, int64_t m, int n, int cnt) {
    if constexpr (is_q8(EPI)) row_scale = a.row_scale[m];
    if constexpr (EPI == MM_PLAIN) {
      if (a.add) g.template load_some<PART>(static_cast<const T*>(a.add) + m * a.ldadd + n, cnt);
    }
    if constexpr (EPI == MM_GATE_BWD) {
      const float* p = a.pre + m * a.ldpre + n;
      g.template load_some<PART>(p, cnt);
      u.template load_some<PART>(p + a.N, cnt);
    }
  }
};

// The columns behind a row of an output whose rows are padded to 16 bytes
// (there are some only if the row ends in a partial piece of 8 columns).
template <typename T>
__device__ __forceinline__ void zero_pad(const MmArgs& a, T* p) {
#pragma unroll 1
  for (int i = 0; i < a.pad; ++i) p[i] = (T)0;
}

// The outputs n .. n + 7 (PART: the first cnt) of row m from the sums c (gated:
// gate sums c, up sums u), which are consumed.
template <int EPI, typename T, bool PART>
__device__ __forceinline__ void finish8(const MmArgs& a, int64_t m, int n, float* c, float* u,
                                        const Cols<EPI, T, PART>& cols, const Extra<EPI, T, PART>& x, int cnt) {
  if constexpr (is_q8(EPI)) {
    cols.gate.apply(a, c, x.row_scale);
    if constexpr (EPI == MM_Q8_GATE) {
      cols.up.apply(a, u, x.row_scale);
      gate8(a.act, c, u);
    }
    if (a.out_f32)
      store_some<PART>(static_cast<float*>(a.out) + m * a.ldo + n, c, cnt);
    else
      store_some<PART>(static_cast<__bf16*>(a.out) + m * a.ldo + n, c, cnt);
  } else if constexpr (EPI == MM_PLAIN) {
    if (a.add) {
      float r[8];
      x.g.get(r);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] += r[i];
    }
    store_some<PART>(static_cast<T*>(a.out) + m * a.ldo + n, c, cnt);
  } else if constexpr (EPI == MM_GATE) {
    if (a.pre) {
      float* p = a.pre + m * a.ldpre + n;
      store_some<PART>(p, c, cnt);
      store_some<PART>(p + a.N, u, cnt);
    }
    gate8(a.act, c, u);
    store_some<PART>(static_cast<T*>(a.out) + m * a.ldo + n, c, cnt);
    if (PART && n + cnt == a.N) zero_pad(a, static_cast<T*>(a.out) + m * a.ldo + a.N);
  } else {
    static_assert(EPI == MM_GATE_BWD);
    float g[8], w[8];
    x.g.get(g);
    x.u.get(w);
    gate8_grad(a.act, c, g, w);
    T* o = static_cast<T*>(a.out) + m * a.ldo + n;
    store_some<PART>(o, g, cnt);
    store_some<PART>(o + a.N, w, cnt);
    if (PART && n + cnt == a.N) zero_pad(a, static_cast<T*>(a.out) + m * a.ldo + 2 * (int64_t)a.N);
  }
}

// finish8 with its reads
template <int EPI, typename T, bool PART>
__device__ __forceinline__ void finish_row(const MmArgs& a, int64_t m, int n, float* c, float* u, int cnt) {
  Cols<EPI, T, PART> cols;
  Extra<EPI, T, PART> x;
  cols.load(a, n, cnt);
  x.load(a, m, n, cnt);
  finish8<EPI, T, PART>(a, m, n, c, u, cols, x, cnt);
}

// Partial sums of a split depth: [split][M][ldp], ldp = N rounded up to 8,
// gated: the up sums in a second such block of columns.
__host__ __device__ __forceinline__ int64_t partial_half(int N) { return ((int64_t)N + 7) / 8 * 8; }
template <int EPI>
__host__ __device__ __forceinline__ int64_t partial_ld(int N) {
  return is_gate(EPI) ? 2 * partial_half(N) : partial_half(N);
}

// One wave's sums acc[i][j], NB x NB blocks of 32 x 32 (rows 32 i + lane % 32,
// columns 32 j + ...), to the outputs: through 4 NB^2 KB of LDS, so that a wave
// reads and writes whole pieces of rows.  A stage row is 8 NB chunks of 16
// bytes, chunk c of row r stored at c ^ (r & (8 NB - 1)).  Gated: the first
// half of the columns are gate sums, the second the up sums of the same
// outputs.
template <int NB>
__device__ __forceinline__ const char* chunk_at(const char* stage, int row, int c) {
  return stage + row * (128 * NB) + ((c ^ (row & (8 * NB - 1))) << 4);
}
template <typename acc_t, int NB, typename A16>
__device__ __forceinline__ void stage_block(const A16 (&acc)[NB][NB], char* stage, int lane) {
  typedef acc_t acc4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const A16& b = acc[i][j];
        *reinterpret_cast<acc4*>(
            const_cast<char*>(chunk_at<NB>(stage, 32 * i + (lane & 31), 8 * j + 2 * q + (lane >> 5)))) =
            acc4{b[4 * q], b[4 * q + 1], b[4 * q + 2], b[4 * q + 3]};
      }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// 8 sums of a row from the stage, from chunk c on
template <int NB>
__device__ __forceinline__ void unstage8(const char* stage, int row, int c, float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(chunk_at<NB>(stage, row, c + h));
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * h + e] = x[e];
  }
}
// Chunk ch of a staged block's rows row, row + RP, ...: outputs n .. n + 7
// (PART: cnt of them) of the rows m, m + RP, ... of C.  What the rows read
// besides the sums is asked for NT rows together.
template <int EPI, typename T, int NB, int NT, bool PART>
__device__ __forceinline__ void write_rows(const MmArgs& a, const char* stage, int m, int row, int n, int ch, int cnt) {
  constexpr int ROWS = 32 * NB, COLS = is_gate(EPI) ? 16 * NB : 32 * NB, RP = 64 / (COLS / 8);
  Cols<EPI, T, PART> cols;
  cols.load(a, n, cnt);
#pragma unroll 1
  for (; row < ROWS; row += NT * RP, m += NT * RP) {
    Extra<EPI, T, PART> x[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) x[b].load(a, min(m + b * RP, a.M - 1), n, cnt);
#pragma unroll
    for (int b = 0; b < NT; ++b) {
      float c[8], u[8];
      unstage8<NB>(stage, row + b * RP, 2 * ch, c);
      if constexpr (is_gate(EPI)) unstage8<NB>(stage, row + b * RP, COLS / 4 + 2 * ch, u);
      if (m + b * RP < a.M) finish8<EPI, T, PART>(a, m + b * RP, n, c, u, cols, x[b], cnt);
    }
  }
}
// The staged block to the outputs; m0, n0: its first row and output column.
template <int EPI, typename T, int NB>
__device__ __forceinline__ void write_block(const MmArgs& a, const char* stage, int m0, int n0, int split, int lane) {
  constexpr int ROWS = 32 * NB, COLS = is_gate(EPI) ? 16 * NB : 32 * NB;
  constexpr int CH = COLS / 8, RP = 64 / CH, NP = ROWS / RP;  // chunks of 8 columns, rows a pass, passes
  const int ch = lane % CH, r0 = lane / CH;
  const int n = n0 + 8 * ch;
  if (a.splits > 1) {
#pragma unroll 1
    for (int it = 0; it < NP; ++it) {
      const int row = it * RP + r0;
      if (n < a.N && m0 + row < a.M) {
        float c[8];
        float* p = a.work + ((int64_t)split * a.M + m0 + row) * partial_ld<EPI>(a.N) + n;
        unstage8<NB>(stage, row, 2 * ch, c);
        store8(p, c);
        if constexpr (is_gate(EPI)) {
          unstage8<NB>(stage, row, COLS / 4 + 2 * ch, c);
          store8(p + partial_half(a.N), c);
        }
      }
    }
  } else if (n + 8 <= a.N) {
    write_rows<EPI, T, NB, NP < 4 ? NP : 4, false>(a, stage, m0 + r0, r0, n, ch, 8);
  } else if (n < a.N) {
    write_rows<EPI, T, NB, 1, true>(a, stage, m0 + r0, r0, n, ch, a.N - n);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Two products in one launch.
struct MmPair {
  MmArgs a, b;
  uint32_t na, nb;  // workgroups of each
};

// The sums of a split depth, joined in order of the splits, by block `block` of
// `blocks`.
template <int EPI, typename T>
__device__ __forceinline__ void join(const MmArgs& a, uint32_t block, uint32_t blocks) {
  const int64_t half = partial_half(a.N), chunks = half / 8, total = a.M * chunks;
  const int64_t ldp = partial_ld<EPI>(a.N);
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < total; i += (int64_t)blocks * 256) {
    const int64_t m = i / chunks;
    const int n = (int)(i % chunks) * 8;
    const float* p = a.work + m * ldp + n;
    float c[8], u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = u[e] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s, p += (int64_t)a.M * ldp) {
      Raw8<float> v, w;
      float f[8], g[8];
      v.load(p);
      v.get(f);
      if constexpr (is_gate(EPI)) {
        w.load(p + half);
        w.get(g);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (is_q8(EPI)) {
          c[e] = __builtin_bit_cast(float, __builtin_bit_cast(int32_t, c[e]) + __builtin_bit_cast(int32_t, f[e]));
          if constexpr (is_gate(EPI))
            u[e] = __builtin_bit_cast(float, __builtin_bit_cast(int32_t, u[e]) + __builtin_bit_cast(int32_t, g[e]));
        } else {
          c[e] += f[e];
          if constexpr (is_gate(EPI)) u[e] += g[e];
        }
      }
    }
    if (n + 8 <= a.N)
      finish_row<EPI, T, false>(a, m, n, c, u, 8);
    else
      finish_row<EPI, T, true>(a, m, n, c, u, a.N - n);
  }
}
template <int EPI, typename T>
__global__ __launch_bounds__(256) void join_kernel(MmArgs a) {
  join<EPI, T>(a, blockIdx.x, gridDim.x);
}
// Both products of a pair: a second launch would cost 4 us, most of it its own
// start (300 tokens of 37, hidden 301, fp32: a training step 50.6 us -> 47.6).
template <int EPI, typename T>
__global__ __launch_bounds__(256) void join_pair_kernel(MmPair p) {
  if (blockIdx.x < p.na)
    join<EPI, T>(p.a, blockIdx.x, p.na);
  else
    join<MM_PLAIN, T>(p.b, blockIdx.x - p.na, p.nb);
}

// ------------------------------------------------------------------ loaders --
// Straight to LDS (base and rows at 16 bytes, the contiguous extent a multiple
// of 16 bytes or zeros behind it up to one): a region of R rows is R / 8 blocks of 1 KB, one load instruction
// each; wave w of NW issues blocks w PER .. w PER + PER - 1.  grow(r): the operand's row
// (rows-contiguous: element) that region row r holds, relative to P, or -1.
// Lanes outside the operand have an offset past the descriptor's range and
// read zeros, so depth past the end adds nothing.
template <int NW, int ES, bool RM, int R = 128>
struct Dma {
  static constexpr int PER = R / 8 / NW;
  const char* base;
  __amdgpu_buffer_rsrc_t rsrc;
  int64_t ldb;
  uint32_t voff[PER];
  int kofs[PER];  // depth of the lane's vector inside a step
  int blk0;
  template <typename F>
  __device__ __forceinline__ void init(const void* P, int64_t ld, int wave, int lane, F grow) {
    base = static_cast<const char*>(P);
    ldb = ld * ES;
    rsrc = make_rsrc(base, kOob);
    blk0 = wave * PER;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int b = blk0 + p;
      if constexpr (!RM) {
        const int row = b * 8 + lane / 8;
        const int c = (lane % 8) ^ kmaj_f<4>(row);
        const int64_t g = grow(row);
        kofs[p] = c * (16 / ES);
        voff[p] = g < 0 ? kOob : (uint32_t)(g * ldb + c * 16);
      } else {
        constexpr int LPK = R * ES / 16;  // lanes a depth row
        const int k = b * (64 / LPK) + lane / LPK;
        // (fp32 is read by consecutive lanes in consecutive banks: no swizzle)
        const int col = ES == 4 ? (lane % LPK) * 4
                                : ((((lane % LPK) >> 1) ^ rmaj_x<R>(k)) << 4) + (lane & 1) * 8;
        const int64_t g = grow(col);
        kofs[p] = k;
        voff[p] = g < 0 ? kOob : (uint32_t)(k * ldb + g * ES);
      }
    }
  }
  // block p of the region at `lds` with the step that starts at depth k0
  __device__ __forceinline__ void issue(char* lds, int64_t k0, int64_t kend, int p) const {
    const uint32_t v = k0 + kofs[p] < kend ? voff[p] : kOob;
    if constexpr (!RM)
      dma16(rsrc, lds + (blk0 + p) * 1024, v, (uint32_t)(k0 * ES));
    else
      dma16(make_rsrc(base + k0 * ldb, kOob), lds + (blk0 + p) * 1024, v, 0);
  }
};

// 16 bytes of global memory at any alignment
__device__ __forceinline__ u32x4 load16(const void* p) {
  return *(const TABPACK_GLOBAL u32x4_any*)p;
}

// Through registers (any alignment and extent): R / 32 vectors of 16 bytes per
// thread of 256 and region.  rbound: rows-contiguous operands end there.
template <typename T, bool RM, int R = 128>
struct Reg {
  static constexpr int VE = Ty<T>::VE, NV = R / 32;
  static constexpr int VPR = RM ? R / VE : 8;  // vectors per line of the region
  const T* base;
  int64_t ld;
  int64_t row[NV];  // operand row (rows-contiguous: element) of the vector, or -1
  int64_t rbound;
  u32x4 v[2][NV];  // two K steps
  template <typename F>
  __device__ __forceinline__ void init(const void* P, int64_t ld_, int64_t rbound_, int tid, F grow) {
    base = static_cast<const T*>(P);
    ld = ld_;
    rbound = rbound_;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int q = tid + i * 256;
      row[i] = RM ? grow((q % VPR) * VE) : grow(q / VPR);
    }
  }
  template <int S>
  __device__ __forceinline__ void load(int64_t k0, int64_t kend, int tid) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int q = tid + i * 256;
      v[S][i] = u32x4{0, 0, 0, 0};
      int64_t left;  // elements of the vector that exist
      const T* p;
      if constexpr (RM) {
        const int64_t k = k0 + q / VPR;
        left = row[i] < 0 || k >= kend ? 0 : rbound - row[i];
        p = base + k * ld + row[i];
      } else {
        const int64_t k = k0 + (q % VPR) * VE;
        left = row[i] < 0 ? 0 : kend - k;
        p = base + row[i] * ld + k;
      }
      if (left >= VE) {
        v[S][i] = load16(p);
      } else if (left > 0) {
        T e[VE];
#pragma unroll
        for (int j = 0; j < VE; ++j) e[j] = j < left ? p[j] : (T)0;
        __builtin_memcpy(&v[S][i], e, 16);
      }
    }
  }
  template <int S>
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int q = tid + i * 256;
      int off;
      if constexpr (!RM)
        off = kmaj16_off<4>(q / VPR, q % VPR);
      else if constexpr (sizeof(T) == 2)
        off = rmaj_off<R>(q / VPR, (q % VPR) * VE);
      else
        off = (q / VPR) * (4 * R) + (q % VPR) * 16;
      *reinterpret_cast<u32x4*>(lds + off) = v[S][i];
    }
  }
};

// -------------------------------------------------------------------- MFMAs --
// acc += (B fragment) (A fragment): lane's values are 4 consecutive columns
// (B rows) of C row lane % 32.
__device__ __forceinline__ void mma(bf16x8 b, bf16x8 a, f32x16& acc, __bf16) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(bf16x8 b, bf16x8 a, i32x16& acc, int8_t) {
  acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, b), __builtin_bit_cast(i32x4, a), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(bf16x8 b, bf16x8 a, f32x16& acc, float) {
  const f32x4 x = __builtin_bit_cast(f32x4, b), y = __builtin_bit_cast(f32x4, a);
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
}

// The 16 bytes that lane needs of rows row .. row + 31 of a region for MFMA
// step ks of 4, in inline assembly (see gemm_tiles.h): the caller waits.
template <typename T, bool RM, int R>
__device__ __forceinline__ bf16x8 frag_asm(const char* lds, int row, int ks, int lane) {
  if constexpr (!RM) {
    return frag_kmaj_asm<4>(lds, row, ks, lane);
  } else if constexpr (sizeof(T) == 2) {
    return frag_tr_asm<R>(lds, row, ks, lane);
  } else {  // fp32 [32 depth rows][R]: depth 8 ks + 4 (lane / 32) .. + 3 of one row, two to an instruction
    typedef __attribute__((address_space(3))) const char* lds_cptr;
    const uint32_t at = (uint32_t)(uintptr_t)(lds_cptr)(lds + (8 * ks + 4 * (lane >> 5)) * (4 * R) +
                                                       (row + (lane & 31)) * 4);
    u32x2 x, y;
    asm volatile("ds_read2st64_b32 %0, %1 offset0:0 offset1:%2" : "=v"(x) : "v"(at), "n"(R / 64));
    asm volatile("ds_read2st64_b32 %0, %1 offset0:%2 offset1:%3" : "=v"(y) : "v"(at), "n"(R / 32), "n"(R / 64 * 3));
    return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
  }
}
// The same as ordinary reads, for regions that were written through registers.
template <typename T, bool RM, int R>
__device__ __forceinline__ bf16x8 frag_reg(const char* lds, int row, int ks, int lane) {
  if constexpr (!RM) {
    return *reinterpret_cast<const bf16x8*>(lds + kmaj16_off<4>(row + (lane & 31), 2 * ks + (lane >> 5)));
  } else if constexpr (sizeof(T) == 2) {
    const int s = lane & 15, g = lane >> 4;
    const int k = 16 * ks + 8 * (g >> 1) + (s >> 2);
    const int col = row + 16 * (g & 1) + 4 * (s & 3);
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + rmaj_off<R>(k, col)));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + rmaj_off<R>(k + 4, col)));
    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
    return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
  } else {  // fp32 [32 depth rows][R]
    f32x4 f;
    const int k = 8 * ks + 4 * (lane >> 5);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      f[e] = *reinterpret_cast<const float*>(lds + (k + e) * (4 * R) + (row + (lane & 31)) * 4);
    return __builtin_bit_cast(bf16x8, f);
  }
}

// Every LDS read of this wave but the last N is done; the fragments named are
// tied to the wait, so no use of them moves before it.
template <int N, int NB>
__device__ __forceinline__ void wait_lds(bf16x8 (&a)[NB], bf16x8 (&b)[NB]) {
  if constexpr (NB == 2)
    asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(a[0]), "+v"(a[1]), "+v"(b[0]), "+v"(b[1]) : "n"(N < 15 ? N : 15));
  else
    asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a[0]), "+v"(b[0]) : "n"(N < 15 ? N : 15));
}

template <typename A16>
__device__ __forceinline__ void clear(A16& a) {
#pragma unroll
  for (int r = 0; r < 16; ++r) a[r] = 0;
}

// The output tile and split of a workgroup.  Workgroups go round the 8 XCDs;
// each XCD gets a contiguous range of tiles (its L2 then holds the panels that
// neighbouring tiles share), walked in bands of 4 tile rows.
struct Where {
  int tm, tn, split;
};
__device__ __forceinline__ Where where(const MmArgs& a, uint32_t block) {
  const uint32_t per = (uint32_t)a.tiles_m * a.tiles_n;
  Where w;
  w.split = block / per;
  const uint32_t b = block % per, q = per / 8, r = per % 8, x = b % 8;
  const uint32_t t = x * q + (x < r ? x : r) + b / 8;
  const uint32_t band = t / (4 * a.tiles_n), in = t % (4 * a.tiles_n);
  const uint32_t h = min(4u, (uint32_t)a.tiles_m - 4 * band);
  w.tm = 4 * band + in % h;
  w.tn = in / h;
  return w;
}

// ---------------------------------------------------- small and mini tiles --
// 64 NB x 64 NB tiles on 4 waves (2 x 2) of NB x NB 32 x 32 blocks.
template <typename T, bool RA, bool RB, int EPI, bool DMA, int NB, int NS>
__device__ __forceinline__ void small_tile(const MmArgs& a, uint32_t block, char* smem) {
  constexpr int ES = sizeof(T), KE = kStep / ES, R = 64 * NB, REGION = R * kStep, W = 32 * NB;
  static_assert(DMA || NS == 2, "two stages through registers");
  typedef typename Ty<T>::acc16 acc16;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const Where w = where(a, block);
  const int m0 = w.tm * R, n0 = w.tn * (is_gate(EPI) ? R / 2 : R);
  const int64_t kbeg = (int64_t)w.split * a.steps_per_split * KE;
  const int64_t kend = min((int64_t)a.K, kbeg + (int64_t)a.steps_per_split * KE);
  const int nk = (int)((kend - kbeg + KE - 1) / KE);
  auto grow_a = [&](int r) -> int64_t { return m0 + r < a.M ? r : -1; };
  // region row of B wn W + x: plain column n0 + that; gated: x < W / 2 the gate
  // row of output n0 + wn W / 2 + x, the others the up rows of the same outputs
  auto grow_b = [&](int r) -> int64_t {
    if constexpr (!is_gate(EPI)) return n0 + r < a.N ? r : -1;
    const int x = (r / W) * (W / 2) + r % (W / 2);
    return n0 + x < a.N ? x + ((r % W) >= W / 2 ? (int64_t)a.N : 0) : -1;
  };
  const T* A = static_cast<const T*>(a.A) + (RA ? (int64_t)m0 : m0 * a.lda);
  const T* B = static_cast<const T*>(a.B) + (RB ? (int64_t)n0 : n0 * a.ldb);
  acc16 acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) clear(acc[i][j]);
  if constexpr (DMA) {
    Dma<4, ES, RA, R> la;
    Dma<4, ES, RB, R> lb;
    la.init(A, a.lda, wave, lane, grow_a);
    lb.init(B, a.ldb, wave, lane, grow_b);
    auto issue = [&](char* st, int64_t k0, int q) {  // quarter q of a step's loads
#pragma unroll
      for (int p = 0; p < NB; ++p) {
        if (q < 2)
          la.issue(st, k0, kend, q * NB + p);
        else
          lb.issue(st + REGION, k0, kend, (q - 2) * NB + p);
      }
    };
    constexpr int NRD = (RA ? 2 * NB : NB) + (RB ? 2 * NB : NB);  // LDS reads per MFMA step
#pragma unroll
    for (int st = 0; st < NS - 1; ++st)
#pragma unroll
      for (int q = 0; q < 4; ++q) issue(smem + st * 2 * REGION, kbeg + (int64_t)st * KE, q);
    int at = 0;  // this step's stage
#pragma unroll 1
    for (int kt = 0; kt < nk; ++kt) {
      char* const cur = smem + at * 2 * REGION;
      wait_vm<(NS - 2) * 4 * NB, true>();
      bar();  // this step has landed, and every wave is done with the last one, whose stage is asked for again
      char* const ahead = smem + (at ? at - 1 : NS - 1) * 2 * REGION;
      at = at + 1 < NS ? at + 1 : 0;
      if constexpr (NS == 2) {
#pragma unroll
        for (int q = 0; q < 4; ++q) issue(ahead, kbeg + (int64_t)(kt + 1) * KE, q);
      }
      bf16x8 fa[4][NB], fb[4][NB];
      auto rd = [&](int ks) {
#pragma unroll
        for (int i = 0; i < NB; ++i) fa[ks][i] = frag_asm<T, RA, R>(cur, wm * W + i * 32, ks, lane);
#pragma unroll
        for (int j = 0; j < NB; ++j) fb[ks][j] = frag_asm<T, RB, R>(cur + REGION, wn * W + j * 32, ks, lane);
      };
      rd(0);
      rd(1);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        if (ks + 2 < 4) rd(ks + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (ks < 2)
          wait_lds<2 * NRD>(fa[ks], fb[ks]);
        else if (ks == 2)
          wait_lds<NRD>(fa[ks], fb[ks]);
        else
          wait_lds<0>(fa[ks], fb[ks]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) mma(fb[ks][j], fa[ks][i], acc[i][j], T());
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (NS > 2) {
          // (with steps to spare the loads go between the products: in one burst
          // they fill the address unit's queue and hold the reads up)
          issue(ahead, kbeg + (int64_t)(kt + NS - 1) * KE, ks);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  } else {
    Reg<T, RA, R> la;
    Reg<T, RB, R> lb;
    la.init(A, a.lda, a.M - m0, tid, grow_a);
    lb.init(B, a.ldb, a.N - n0, tid, grow_b);
    // step kt, whose vectors are in register set and LDS stage S; set S takes step kt + 2
    auto step = [&](auto set, int kt) {
      constexpr int S = decltype(set)::value;
      char* const cur = smem + S * 2 * REGION;
      la.template store<S>(cur, tid);
      lb.template store<S>(cur + REGION, tid);
      __syncthreads();  // the other stage was read before the barrier of the step before this one's stores
      la.template load<S>(kbeg + (int64_t)(kt + 2) * KE, kend, tid);
      lb.template load<S>(kbeg + (int64_t)(kt + 2) * KE, kend, tid);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        bf16x8 fa[NB], fb[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) fa[i] = frag_reg<T, RA, R>(cur, wm * W + i * 32, ks, lane);
#pragma unroll
        for (int j = 0; j < NB; ++j) fb[j] = frag_reg<T, RB, R>(cur + REGION, wn * W + j * 32, ks, lane);
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) mma(fb[j], fa[i], acc[i][j], T());
      }
    };
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;
    la.template load<0>(kbeg, kend, tid);
    lb.template load<0>(kbeg, kend, tid);
    la.template load<1>(kbeg + KE, kend, tid);
    lb.template load<1>(kbeg + KE, kend, tid);
#pragma unroll 1
    for (int kt = 0; kt < nk; kt += 2) {
      step(S0{}, kt);
      if (kt + 1 < nk) step(S1{}, kt + 1);
    }
  }
  wait_vm<0, true>();
  bar();  // the sums are staged in the operand regions
  char* const stage = smem + wave * (4096 * NB * NB);
  stage_block<typename Ty<T>::acc_t, NB>(acc, stage, lane);
  write_block<EPI, T, NB>(a, stage, m0 + wm * W, n0 + wn * (is_gate(EPI) ? W / 2 : W), w.split, lane);
}

// -------------------------------------------------------------- huge tiles --
// LDS addresses of a wave's fragments of one operand inside a region; what is
// a constant distance goes into the instruction's offset.  Depth-contiguous:
// v[ks], row block i 4 KB on (32 rows do not change the swizzle).
// Rows-contiguous: v[i], MFMA step ks 4 KB on.
template <bool RM, int NI>
struct FragAddr {
  uint32_t v[RM ? NI : 4];
  __device__ __forceinline__ void init(const char* lds, int row0, int lane) {
    typedef __attribute__((address_space(3))) const char* lds_cptr;
    const uint32_t base = (uint32_t)(uintptr_t)(lds_cptr)lds;
    if constexpr (!RM) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) v[ks] = base + kmaj16_off<4>(row0 + (lane & 31), 2 * ks + (lane >> 5));
    } else {
      const int s = lane & 15, g = lane >> 4;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        v[i] = base + rmaj_off<128>(8 * (g >> 1) + (s >> 2), row0 + 32 * i + 16 * (g & 1) + 4 * (s & 3));
    }
  }
  template <int I, int KS>
  __device__ __forceinline__ void read(bf16x8& f, uint32_t region) const {
    if constexpr (!RM) {
      u32x4 r;
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(v[KS] + region), "n"(I * 4096));
      f = __builtin_bit_cast(bf16x8, r);
    } else {
      u32x2 x, y;
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(x) : "v"(v[I] + region), "n"(KS * 4096));
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(y) : "v"(v[I] + region), "n"(KS * 4096 + 1024));
      f = __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
    }
  }
  // the fragments of row block I of the region at byte `region`
  template <int I>
  __device__ __forceinline__ void read4(bf16x8 (&f)[4], uint32_t region) const {
    read<I, 0>(f[0], region);
    read<I, 1>(f[1], region);
    read<I, 2>(f[2], region);
    read<I, 3>(f[3], region);
  }
};
__device__ __forceinline__ void tie(bf16x8 (&f)[4]) {
  asm volatile("" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]));
}

// A wave's 128 x 64 sums to the outputs, one 64 x 64 half after the other.  No
// other workgroup on the CU covers the waits, so what a piece's rows read besides
// the sums is asked for a piece ahead: 32 rows, or 16 where they read two fp32
// values an output (32 would not fit the registers).
template <int EPI, typename T, typename A16>
__device__ __forceinline__ void huge_out(const MmArgs& a, const A16 (&acc)[2][2][2], char* stage, int m0, int n0,
                                         int split, int lane) {
  typedef typename Ty<T>::acc_t acc_t;
  constexpr int COLS = is_gate(EPI) ? 32 : 64, CH = COLS / 8, RP = 64 / CH;
  constexpr int PIECE = EPI == MM_GATE_BWD ? 16 : 32, PIECES = 64 / PIECE, NP = PIECE / RP;  // NP passes a piece
  const int ch = lane % CH, r0 = lane / CH, n = n0 + 8 * ch;
  if (a.splits > 1 || n0 + COLS > a.N) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      stage_block<acc_t, 2>(acc[h], stage, lane);
      write_block<EPI, T, 2>(a, stage, m0 + h * 64, n0, split, lane);
    }
    return;
  }
  Cols<EPI, T, false> cols;
  cols.load(a, n, 8);
  Extra<EPI, T, false> x[NP], y[NP];
  auto ask = [&](Extra<EPI, T, false>(&e)[NP], int q) {
#pragma unroll
    for (int p = 0; p < NP; ++p) e[p].load(a, min(m0 + q * PIECE + p * RP + r0, a.M - 1), n, 8);
  };
  ask(x, 0);
#pragma unroll
  for (int h = 0; h < 2; ++h) {  // (unrolled: the first half's sums give up their registers)
    stage_block<acc_t, 2>(acc[h], stage, lane);
#pragma unroll 1
    for (int q = 0; q < PIECES; ++q) {
      if (PIECES * h + q + 1 < 2 * PIECES) ask(y, PIECES * h + q + 1);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int row = q * PIECE + p * RP + r0, m = m0 + h * 64 + row;
        float c[8], u[8];
        unstage8<2>(stage, row, 2 * ch, c);
        if constexpr (is_gate(EPI)) unstage8<2>(stage, row, 8 + 2 * ch, u);
        if (m < a.M) finish8<EPI, T, false>(a, m, n, c, u, cols, x[p], 8);
      }
#pragma unroll
      for (int p = 0; p < NP; ++p) x[p] = y[p];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// 256 x 256 tiles on 8 waves (2 x 4, two to a SIMD), each 128 x 64.  A K step
// is two phases, one half (64 x 64) of the wave's sums each; a phase is a read
// part (the half's fragments from LDS) and a product part (16 MFMAs, with the
// loads of later steps between them), with a barrier after each.  The waves of
// the tile's lower half run one part behind those of the upper half, so on
// every SIMD one wave's products run beside the other's reads; the wave with
// products has priority.
// The 16 KB regions are numbered A half 0, B half 0, B half 1, A half 1 of step
// 0, of step 1, ...: region n lies in slot n % 10 of LDS; phase g asks for the
// regions 2 g + 8 and 2 g + 9.  When the reads of phase g end, those up to 2 g +
// 7 have been asked for and the next phase needs region 2 g + 3 (g even) or
// 2 g + 4: the newest 4 or 3 may be in flight, vmcnt(8) or (6) (two loads a
// region and wave) before the barrier.  A slot is asked for again in the phase
// after its last reads at the earliest, in the product part, when the lagging
// waves have finished theirs.
constexpr int kHugeSlots = 10;
template <typename T, bool RA, bool RB, int EPI>
__device__ __forceinline__ void huge_tile(const MmArgs& a, uint32_t block, char* smem) {
  constexpr int ES = sizeof(T), KE = kStep / ES, SLOTS = kHugeSlots;
  typedef typename Ty<T>::acc16 acc16;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const Where w = where(a, block);
  const int m0 = w.tm * 256, n0 = w.tn * (is_gate(EPI) ? 128 : 256);
  const int64_t kbeg = (int64_t)w.split * a.steps_per_split * KE;
  const int64_t kend = min((int64_t)a.K, kbeg + (int64_t)a.steps_per_split * KE);
  const int nk = (int)((kend - kbeg + KE - 1) / KE);
  const T* A = static_cast<const T*>(a.A) + (RA ? (int64_t)m0 : m0 * a.lda);
  const T* B = static_cast<const T*>(a.B) + (RB ? (int64_t)n0 : n0 * a.ldb);
  Dma<8, ES, RA> la[2];
  Dma<8, ES, RB> lb[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // A half h: the rows of phases 2h, 2h + 1 of both wave rows; B half h: the
    // columns of two phases of every wave column (gated: gate rows, up rows)
    la[h].init(A, a.lda, wave, lane, [&](int r) -> int64_t {
      const int x = (r >> 6) * 128 + h * 64 + (r & 63);
      return m0 + x < a.M ? x : -1;
    });
    lb[h].init(B, a.ldb, wave, lane, [&](int r) -> int64_t {
      if constexpr (is_gate(EPI)) return n0 + r < a.N ? r + (h ? (int64_t)a.N : 0) : -1;
      const int x = (r >> 5) * 64 + h * 32 + (r & 31);
      return n0 + x < a.N ? x : -1;
    });
  }
  auto ask_a = [&](int h, int step, int slot, int p) {
    la[h].issue(smem + slot * kRegion, kbeg + (int64_t)step * KE, kend, p);
  };
  auto ask_b = [&](int h, int step, int slot, int p) {
    lb[h].issue(smem + slot * kRegion, kbeg + (int64_t)step * KE, kend, p);
  };
  FragAddr<RA, 2> fa;
  FragAddr<RB, 1> fb;
  fa.init(smem, wm * 64, lane);
  fb.init(smem, wn * 32, lane);
  acc16 acc[2][2][2];  // [A half][32-row block][B half]
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) clear(acc[h][i][j]);
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      if (n % 4 == 0 || n % 4 == 3)
        ask_a(n % 4 == 3, n / 4, n, p);
      else
        ask_b(n % 4 == 2, n / 4, n, p);
    }
  wait_vm<10, false>();
  bar();
  if (wm == 1) bar();
  bf16x8 x0[4], x1[4], y0[4], y1[4];  // A row blocks 0 and 1 of the half; B halves
  // end of a phase's reads, and its products
  auto products = [&](acc16 (&c)[2][2], auto vm, auto ask) {
    __builtin_amdgcn_sched_barrier(0);
    wait_vm<decltype(vm)::value, false>();
    bar();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    tie(x0);
    tie(x1);
    tie(y0);
    tie(y1);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      mma(y0[ks], x0[ks], c[0][0], T());
      mma(y0[ks], x1[ks], c[1][0], T());
      mma(y1[ks], x0[ks], c[0][1], T());
      __builtin_amdgcn_sched_barrier(0);
      ask(ks);
      __builtin_amdgcn_sched_barrier(0);
      mma(y1[ks], x1[ks], c[1][1], T());
    }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    bar();
  };
  int slot = 0;  // of the step's first region
  auto after = [](int sl, int n) { return sl + n < SLOTS ? sl + n : sl + n - SLOTS; };
#pragma unroll 1
  for (int kt = 0; kt < nk; ++kt) {
    fa.template read4<0>(x0, slot * kRegion);
    fa.template read4<1>(x1, slot * kRegion);
    fb.template read4<0>(y0, after(slot, 1) * kRegion);
    fb.template read4<0>(y1, after(slot, 2) * kRegion);
    products(acc[0], std::integral_constant<int, 8>{}, [&](int q) {
      if (q < 2)
        ask_a(0, kt + 2, after(slot, 8), q);
      else
        ask_b(0, kt + 2, after(slot, 9), q - 2);
    });
    fa.template read4<0>(x0, after(slot, 3) * kRegion);
    fa.template read4<1>(x1, after(slot, 3) * kRegion);
    products(acc[1], std::integral_constant<int, 6>{}, [&](int q) {
      if (q < 2)
        ask_b(1, kt + 2, slot, q);
      else
        ask_a(1, kt + 2, after(slot, 1), q - 2);
    });
    slot = after(slot, 4);
  }
  if (wm == 0) bar();
  wait_vm<0, true>();
  bar();  // the sums are staged in the operand regions
  huge_out<EPI, T>(a, acc, smem + wave * 16384, m0 + wm * 128, n0 + wn * (is_gate(EPI) ? 32 : 64), w.split, lane);
}

// ----------------------------------------------------------------- kernels --
// One product, or two independent ones in one launch, which fill the chip
// together where each alone leaves CUs idle: b's workgroups spread evenly among
// a's in octets (an octet covers the XCDs).  The part of the launch that this
// workgroup has: product 0 or 1 (2: none).
__device__ __forceinline__ int part_of(const MmPair& p, uint32_t& block) {
  const uint32_t oa = (p.na + 7) / 8, ob = (p.nb + 7) / 8, o = blockIdx.x / 8;
  const uint32_t lo = (uint32_t)((uint64_t)o * ob / (oa + ob)), hi = (uint32_t)(((uint64_t)o + 1) * ob / (oa + ob));
  const bool second = hi > lo;
  block = (second ? lo : o - lo) * 8 + blockIdx.x % 8;
  return second ? (block < p.nb ? 1 : 2) : (block < p.na ? 0 : 2);
}

template <typename T, bool RA, bool RB, int EPI, bool DMA, int NB, int NS>
__global__ __launch_bounds__(256, NB * NS == 4 ? 2 : 4) void small_kernel(MmArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[2 * NS * 64 * NB * kStep];
  small_tile<T, RA, RB, EPI, DMA, NB, NS>(a, blockIdx.x, smem);
}
template <typename T, int EPI, bool DMA, int NB, int NS>
__global__ __launch_bounds__(256, NB * NS == 4 ? 2 : 4) void small_pair_kernel(MmPair p) {
  __shared__ __attribute__((aligned(16))) char smem[2 * NS * 64 * NB * kStep];
  uint32_t block;
  const int part = part_of(p, block);
  if (part == 0)
    small_tile<T, false, true, EPI, DMA, NB, NS>(p.a, block, smem);
  else if (part == 1)
    small_tile<T, true, true, MM_PLAIN, DMA, NB, NS>(p.b, block, smem);
}
template <typename T, bool RA, bool RB, int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void huge_kernel(MmArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kHugeSlots * kRegion];
  huge_tile<T, RA, RB, EPI>(a, blockIdx.x, smem);
}
// -------------------------------------------------------------- thin tiles --
// Up to 16 rows of A (depth-contiguous operands, bf16 and int8): a workgroup
// owns 16 columns (gated: 16 gate and 16 up rows of B), its NW waves share the
// depth in strips of 256 bytes, and every weight byte is read once, straight
// into MFMA operands (16 x 16 blocks; lane l holds 16 bytes of depth of row
// l % 16).  The loads bound it: a strip's are all issued before its products,
// at any alignment.  The waves' sums meet in LDS, added in order.  One row, 4096
// gated outputs, depth 1024: int8 4.0 us (2.1 TB/s of weights, a third of it the
// launch), bf16 5.3; 4096 gated outputs at depth 4096 bf16 14 us (4.7 TB/s).
__device__ __forceinline__ void mma16(u32x4 b, u32x4 a, f32x4& acc, __bf16) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), acc, 0,
                                                0, 0);
}
__device__ __forceinline__ void mma16(u32x4 b, u32x4 a, i32x4& acc, int8_t) {
  acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, b), __builtin_bit_cast(i32x4, a), acc, 0, 0, 0);
}
// 16 bytes of a row from element k on, zeros from kend on
template <typename T>
__device__ __forceinline__ u32x4 row16(const T* row, int64_t k, int64_t kend) {
  constexpr int VE = Ty<T>::VE;
  u32x4 v{0, 0, 0, 0};
  if (k + VE <= kend) {
    v = load16(row + k);
  } else if (k < kend) {
    T e[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) e[j] = k + j < kend ? row[k + j] : (T)0;
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}
template <typename T, int EPI, int NW>
__global__ __launch_bounds__(NW * 64) void thin_kernel(MmArgs a) {
  constexpr int G = is_gate(EPI) ? 2 : 1, ES = sizeof(T), STRIP = 256 / ES, UNIT = 64 / ES;
  typedef typename Ty<T>::acc_t acc_t;
  typedef acc_t acc4 __attribute__((ext_vector_type(4)));
  __shared__ acc4 sums[NW][G][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int64_t K = a.K;
  // rows and columns past the end read the last one; their sums are not used
  const T* wrow[G];
  const T* const xrow = static_cast<const T*>(a.A) + min(lane % 16, a.M - 1) * a.lda;
  const int64_t kl = (lane / 16) * (16 / ES);  // the lane's depth inside a unit
#pragma unroll
  for (int g = 0; g < G; ++g)
    wrow[g] = static_cast<const T*>(a.B) + (min(n0 + lane % 16, a.N - 1) + (int64_t)g * a.N) * a.ldb;
  acc4 acc[G];
#pragma unroll
  for (int g = 0; g < G; ++g) acc[g] = acc4{0, 0, 0, 0};
  struct Strip {
    u32x4 w[G][4], x[4];
  };
  const int64_t strips = (K + STRIP - 1) / STRIP;
  auto load = [&](Strip& f, int64_t st) {
    const int64_t k0 = st * STRIP + kl;
    if ((st + 1) * STRIP <= K) {  // the same for the whole wave
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int g = 0; g < G; ++g) f.w[g][u] = load16(wrow[g] + k0 + u * UNIT);
        f.x[u] = load16(xrow + k0 + u * UNIT);
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int g = 0; g < G; ++g) f.w[g][u] = row16(wrow[g], k0 + u * UNIT, K);
        f.x[u] = row16(xrow, k0 + u * UNIT, K);
      }
    }
  };
  auto products = [&](const Strip& f) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int g = 0; g < G; ++g) mma16(f.w[g][u], f.x[u], acc[g], T());
  };
  // the next strip is asked for before the products of the present one
  if (wave < strips) {
    Strip f, next;
    load(f, wave);
    for (int64_t st = wave; st < strips; st += NW) {
      const bool more = st + NW < strips;
      if (more) load(next, st + NW);
      products(f);
      if (more) f = next;
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) sums[wave][g][lane] = acc[g];
  __syncthreads();
  // lane of the first wave: row lane % 16, columns n0 + 4 (lane / 16) ..  + 3
  const int m = lane % 16, n = n0 + 4 * (lane / 16);
  if (tid >= 64 || m >= a.M) return;
  acc4 c = sums[0][0][lane], u = sums[0][G - 1][lane];
#pragma unroll
  for (int q = 1; q < NW; ++q) {
    c += sums[q][0][lane];
    if constexpr (G == 2) u += sums[q][1][lane];
  }
  if (n >= a.N) return;
  float cs[8], us[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const acc_t ce = c[e & 3], ue = u[e & 3];
    cs[e] = __builtin_bit_cast(float, ce);
    us[e] = __builtin_bit_cast(float, ue);
  }
  finish_row<EPI, T, true>(a, m, n, cs, us, min(4, a.N - n));
}

// ------------------------------------------------------------ aligned copies --
// Matrices whose rows cannot start at 16 bytes or end inside a vector, copied
// to rows of whole 128-byte lines with zeros behind their ends.  G = 1 << g
// lanes a row, four vectors of each lane in flight.  Bandwidth bounds it.
struct CopyArgs {
  const char* src[3];
  char* dst[3];
  int64_t lds[3], ldd[3], width[3];  // bytes between rows, and of a row
  int64_t rows[3];
  uint32_t blocks[3];
  int32_t g[3];
};
__global__ __launch_bounds__(256) void copy_rows_kernel(CopyArgs c) {
  uint32_t block = blockIdx.x;
  int i = 0;
  while (i < 2 && block >= c.blocks[i]) block -= c.blocks[i++];
  const char* const src = c.src[i];
  char* const dst = c.dst[i];
  const int64_t width = c.width[i], rows = c.rows[i], nv = c.ldd[i] / 16;
  const int g = c.g[i], lane = threadIdx.x & ((1 << g) - 1);
  const int64_t step = (int64_t)c.blocks[i] * (256 >> g);
  for (int64_t r = (int64_t)block * (256 >> g) + (threadIdx.x >> g); r < rows; r += step) {
    const char* const p = src + r * c.lds[i];
    u32x4* const q = reinterpret_cast<u32x4*>(dst + r * c.ldd[i]);
    for (int64_t v0 = lane; v0 < nv; v0 += 4 << g) {
      u32x4 x[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int64_t at = (v0 + ((int64_t)b << g)) * 16;
        x[b] = u32x4{0, 0, 0, 0};
        if (at + 16 <= width) {
          x[b] = load16(p + at);
        } else if (at < width) {
          char e[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) e[j] = at + j < width ? p[at + j] : 0;
          __builtin_memcpy(&x[b], e, 16);
        }
      }
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if (v0 + ((int64_t)b << g) < nv) q[v0 + ((int64_t)b << g)] = x[b];
    }
  }
}

// ------------------------------------------------------------------- host --
enum Tiles { TILES_THIN, TILES_MINI, TILES_SMALL, TILES_HUGE };
// How a product is laid out over workgroups.
struct Plan {
  Tiles tiles;
  int64_t tm, tn;
  int splits, steps;  // workgroups that share a tile's depth, K steps of each
  double us;          // the model's time
};

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

int elem_bytes(MmType t) { return t == MM_BF16 ? 2 : t == MM_FP32 ? 4 : 1; }

int64_t depth_steps(MmType type, const MmArgs& a) {
  return a.K > 0 ? cdiv((int64_t)a.K * elem_bytes(type), kStep) : 1;
}

Plan plan_with(MmType type, const MmArgs& a, Tiles t, int64_t splits) {
  const int side = t == TILES_HUGE ? 256 : t == TILES_SMALL ? 128 : 64;
  Plan p;
  p.tiles = t;
  p.tm = t == TILES_THIN ? 1 : cdiv(a.M, side);
  p.tn = t == TILES_THIN ? cdiv(a.N, 16) : cdiv(a.N, is_gate(a.epi) ? side / 2 : side);
  const int64_t steps = depth_steps(type, a);
  splits = std::max((int64_t)1, std::min(splits, steps));
  p.steps = (int)cdiv(steps, splits);
  p.splits = (int)cdiv(steps, p.steps);
  p.us = 0;
  return p;
}

// A model of a product's time in us, fitted to measurements of 128..16384 rows,
// 256..4096 columns and depths 1024..16384 (fewer rows and shorter depths are
// extrapolated): a start, a time per K step that
// grows with the tiles a CU holds, and the join's traffic.  Mini tiles step in
// 0.2 us a tile, small ones in 0.6, huge ones in 1.05 on a few CUs and 1.6 where
// all of them run (the clock falls under their power); operands through
// registers take 0.42 and 0.9, half as much again for each that is
// rows-contiguous; fp32 0.62 and 2.2, through registers 0.7 and 2.45.
double step_us(MmType type, const MmArgs& a, Tiles t, bool dma, double wgs) {
  const double held = std::ceil(wgs / 256);
  if (t == TILES_HUGE) return wgs < 256 ? 1.05 + 0.55 * wgs / 256 : 1.6 * held;
  if (type == MM_FP32)
    return t == TILES_MINI ? (dma ? std::max(0.75, 0.62 * held) : std::max(0.85, 0.7 * held))
                           : (dma ? 2.2 : 2.45) * held;
  if (!dma)
    return (1 + 0.5 * (a.a_rmaj + a.b_rmaj)) *
           (t == TILES_MINI ? std::max(0.55, 0.42 * held) : std::max(1.05, 0.9 * held));
  return (t == TILES_MINI ? 0.2 : 0.6) * held;
}
double start_us(Tiles t) { return t == TILES_HUGE ? 7 : 3.3; }
double join_us(const MmArgs& a, const Plan& p) {
  if (p.splits < 2) return 0;
  return 4 + p.splits * (double)a.M * ((a.N + 7) / 8 * 8) * (is_gate(a.epi) ? 16 : 8) / 3.5e6;
}
constexpr int64_t kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};

// The layout that should be fastest.  Up to 16 rows the thin kernel (at depth
// 1024 and 1024..4096 columns 3.8-5.1 us against 5.6-6.8 on mini tiles; at 32
// rows it no longer gains: 7.0 / 6.6, depth 4096 13.4 / 9.9 split), the others
// by the model.  Thin products of few columns leave CUs idle, whatever their
// depth: 1024 columns are 64 workgroups, at depth 4096 in bf16 7.5 us, 1.1 TB/s of
// weights.
Plan search(MmType type, const MmArgs& a, bool dma) {
  Plan best = plan_with(type, a, TILES_MINI, 1);
  best.us = 1e30;
  if (type != MM_FP32 && !a.a_rmaj && !a.b_rmaj && a.M <= 16) return plan_with(type, a, TILES_THIN, 1);
  for (Tiles t : {TILES_MINI, TILES_SMALL, TILES_HUGE}) {
    if (t == TILES_HUGE && (!dma || type == MM_FP32)) continue;
    int64_t last = 0;
    for (int64_t s : kSplits) {
      Plan p = plan_with(type, a, t, s);
      if (p.splits == last || (p.splits > 1 && p.steps < 2)) continue;
      last = p.splits;
      p.us = start_us(t) + p.steps * step_us(type, a, t, dma, (double)p.tm * p.tn * p.splits) + join_us(a, p);
      if (p.us < best.us) best = p;
    }
  }
  return best;
}

// search(), whose result depends on the sizes alone, with its last answers kept
// (it costs about a microsecond, a block's calls ask for up to 20 plans).
Plan choose(MmType type, const MmArgs& a, bool dma) {
  struct Memo {
    int32_t M, N, K, kind;
    Plan plan;
  };
  static thread_local Memo memo[64];
  const int32_t kind = 1 + (int)type + 4 * a.epi + 32 * a.a_rmaj + 64 * a.b_rmaj + 128 * (int)dma;  // 0: empty
  const uint32_t at = ((uint32_t)a.M * 0x9E3779B1u ^ (uint32_t)a.N * 0x85EBCA77u ^ (uint32_t)a.K * 0xC2B2AE3Du ^
                       (uint32_t)kind * 0x27D4EB2Fu) >> 26;
  Memo& e = memo[at];
  if (e.M != a.M || e.N != a.N || e.K != a.K || e.kind != kind)
    e = Memo{a.M, a.N, a.K, kind, search(type, a, dma)};
  return e.plan;
}

size_t partial_bytes(const MmArgs& a, const Plan& p) {
  if (p.splits < 2) return 0;
  return (size_t)p.splits * (size_t)a.M * (size_t)partial_half(a.N) * (is_gate(a.epi) ? 8 : 4);
}

bool rows16(const void* p, int64_t ld, int es) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0;
}

// Whether an operand's rows in memory end inside a 16-byte vector, with what is
// not a zero behind them.
bool odd_a(MmType type, const MmArgs& a) {
  return !a.a_zero && (int64_t)(a.a_rmaj ? a.M : a.K) * elem_bytes(type) % 16 != 0;
}
bool odd_b(MmType type, const MmArgs& a) {
  return !a.b_zero && (int64_t)(a.b_rmaj ? a.N : a.K) * elem_bytes(type) % 16 != 0;
}

// Whether both operands can go straight to LDS: rows at 16 bytes, whole 16-byte
// vectors, and tile-relative offsets below 2 GiB.
bool can_dma(MmType type, const MmArgs& a) {
  const int es = elem_bytes(type);
  if (odd_a(type, a) || odd_b(type, a) || !rows16(a.A, a.lda, es) || !rows16(a.B, a.ldb, es)) return false;
  const int64_t lim = (int64_t)1 << 31;
  const int64_t brows = is_gate(a.epi) ? (int64_t)a.N + 256 : 256;
  return a.lda * es * 256 < lim && a.ldb * es * brows < lim && (int64_t)a.K * es < lim / 2;
}

template <typename T, int EPI>
void launch_thin(const MmArgs& a, dim3 grid, hipStream_t s) {
  // a wave per 256-byte strip of depth, 4 to 16 of them (gated 8: two strips of
  // two weight rows do not fit the registers of 16)
  constexpr int MOST = is_gate(EPI) ? 8 : 16;
  const int64_t strips = cdiv((int64_t)a.K * (int)sizeof(T), 256);
  if (strips > 8)
    hipLaunchKernelGGL((thin_kernel<T, EPI, MOST>), grid, dim3(MOST * 64), 0, s, a);
  else if (strips > 4)
    hipLaunchKernelGGL((thin_kernel<T, EPI, 8>), grid, dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((thin_kernel<T, EPI, 4>), grid, dim3(256), 0, s, a);
}

// Fills in the launch's part of the arguments; its workgroups (0: too many for a launch).
uint32_t apply(MmArgs& a, const Plan& p) {
  a.tiles_m = (int)p.tm, a.tiles_n = (int)p.tn, a.splits = p.splits, a.steps_per_split = p.steps;
  const int64_t blocks = p.tm * p.tn * p.splits;
  return blocks <= (1 << 22) ? (uint32_t)blocks : 0;  // (a launch is limited to 2^32 threads, m0 to 2^31)
}

// Workgroups that join a product's split depth (0: it is not split).
uint32_t join_blocks(const MmArgs& a) {
  if (a.splits < 2 || !a.out) return 0;
  return (uint32_t)std::min(cdiv((int64_t)a.M * (partial_half(a.N) / 8), 256), (int64_t)4096);
}
template <int EPI, typename T>
void launch_join(const MmArgs& a, hipStream_t s) {
  const uint32_t n = join_blocks(a);
  if (n) hipLaunchKernelGGL((join_kernel<EPI, T>), dim3(n), dim3(256), 0, s, a);
}

template <typename T, bool RA, bool RB, int EPI>
hipError_t launch_tiles(MmType type, MmArgs a, hipStream_t s) {
  const bool dma = can_dma(type, a);
  const Plan p = choose(type, a, dma);
  const dim3 grid(apply(a, p));
  if (grid.x == 0) return hipErrorInvalidConfiguration;
  if (a.work_bytes < partial_bytes(a, p)) return hipErrorInvalidValue;
  if constexpr (sizeof(T) != 4 && !RA && !RB) {
    if (p.tiles == TILES_THIN) {
      launch_thin<T, EPI>(a, grid, s);
      return hipGetLastError();
    }
  }
  if (p.tiles == TILES_HUGE) {
    if constexpr (sizeof(T) != 4) hipLaunchKernelGGL((huge_kernel<T, RA, RB, EPI>), grid, dim3(512), 0, s, a);
  } else if (dma && p.tiles == TILES_SMALL) {
    hipLaunchKernelGGL((small_kernel<T, RA, RB, EPI, true, 2, 2>), grid, dim3(256), 0, s, a);
  } else if (dma) {
    hipLaunchKernelGGL((small_kernel<T, RA, RB, EPI, true, 1, 4>), grid, dim3(256), 0, s, a);
  } else if (p.tiles == TILES_SMALL) {
    hipLaunchKernelGGL((small_kernel<T, RA, RB, EPI, false, 2, 2>), grid, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((small_kernel<T, RA, RB, EPI, false, 1, 2>), grid, dim3(256), 0, s, a);
  }
  launch_join<EPI, T>(a, s);
  return hipGetLastError();
}

// Two products in one launch: the same tiles, and depths split so that the
// workgroups of both take about the same number of steps.  Not for huge tiles:
// the gradients of gate and up beside the down weights' (16,384 tokens of 1024,
// hidden 4096; g and u read in bf16) 365 us together, 222 + 122 apart.
struct PairPlan {
  Plan a, b;
  double us;
};
PairPlan search_pair(MmType type, const MmArgs& a, const MmArgs& b, bool dma) {
  PairPlan best;
  best.us = 1e30;
  const int64_t sa = depth_steps(type, a), sb = depth_steps(type, b);
  for (Tiles t : {TILES_MINI, TILES_SMALL}) {
    for (int64_t s : kSplits) {
      const int64_t q = cdiv(std::max(sa, sb), s);  // most steps of a workgroup
      if (s > 1 && q < 2) break;
      PairPlan p;
      p.a = plan_with(type, a, t, cdiv(sa, q));
      p.b = plan_with(type, b, t, cdiv(sb, q));
      const double wa = (double)p.a.tm * p.a.tn * p.a.splits, wb = (double)p.b.tm * p.b.tn * p.b.splits;
      // the workgroups of a CU one after the other, but no less than the longest one
      const double mean = (wa * p.a.steps + wb * p.b.steps) / (wa + wb);
      const double longest = std::max(p.a.steps, p.b.steps);
      p.us = start_us(t) + join_us(a, p.a) + join_us(b, p.b) +
             std::max(mean * step_us(type, b, t, dma, wa + wb),
                      longest * step_us(type, b, t, dma, std::min(wa + wb, 256.0)));
      if (p.us < best.us) best = p;
    }
  }
  return best;
}
// Whether the two go together (remembered as choose()'s plans are); their
// workspace lies one after the other.
bool pair_up(MmType type, const MmArgs& a, const MmArgs& b, bool dma, PairPlan& p) {
  if (a.M < 1 || b.K < 1) return false;
  struct Memo {
    int32_t size[6], kind;
    PairPlan plan;
    bool good;
  };
  static thread_local Memo memo[16];
  const int32_t size[6] = {a.M, a.N, a.K, b.M, b.N, b.K};
  const int32_t kind = 1 + (int)type + 4 * a.epi + 128 * (int)dma;  // 0: empty
  uint32_t h = (uint32_t)kind;
  for (int32_t v : size) h = (h ^ (uint32_t)v) * 0x9E3779B1u;
  Memo& e = memo[h >> 28];
  if (e.kind != kind || !std::equal(size, size + 6, e.size)) {
    std::copy(size, size + 6, e.size);
    e.kind = kind;
    e.plan = search_pair(type, a, b, dma);
    e.good = e.plan.us < choose(type, a, dma).us + choose(type, b, dma).us;
  }
  p = e.plan;
  return e.good;
}
size_t pair_bytes(const MmArgs& a, const MmArgs& b, const PairPlan& p) {
  return (partial_bytes(a, p.a) + 15) / 16 * 16 + partial_bytes(b, p.b);
}

template <typename T, int EPI>
hipError_t launch_pair(MmType type, MmArgs a, MmArgs b, const PairPlan& p, bool dma, hipStream_t s) {
  MmPair m;
  m.na = apply(a, p.a);
  m.nb = apply(b, p.b);
  if (m.na == 0 || m.nb == 0) return hipErrorInvalidConfiguration;
  if (!a.out) m.na = 0;
  if (!b.out) m.nb = 0;
  if (a.work_bytes < pair_bytes(a, b, p)) return hipErrorInvalidValue;
  b.work += (partial_bytes(a, p.a) + 15) / 16 * 4;
  m.a = a, m.b = b;
  const dim3 grid(((m.na + 7) / 8 + (m.nb + 7) / 8) * 8);
  const Tiles t = p.a.tiles;
  if (dma && t == TILES_SMALL)
    hipLaunchKernelGGL((small_pair_kernel<T, EPI, true, 2, 2>), grid, dim3(256), 0, s, m);
  else if (dma)
    hipLaunchKernelGGL((small_pair_kernel<T, EPI, true, 1, 4>), grid, dim3(256), 0, s, m);
  else if (t == TILES_SMALL)
    hipLaunchKernelGGL((small_pair_kernel<T, EPI, false, 2, 2>), grid, dim3(256), 0, s, m);
  else
    hipLaunchKernelGGL((small_pair_kernel<T, EPI, false, 1, 2>), grid, dim3(256), 0, s, m);
  m.na = join_blocks(a), m.nb = join_blocks(b);
  if (m.na && m.nb) {
    hipLaunchKernelGGL((join_pair_kernel<EPI, T>), dim3(m.na + m.nb), dim3(256), 0, s, m);
  } else {
    launch_join<EPI, T>(a, s);
    launch_join<MM_PLAIN, T>(b, s);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_float(MmType type, const MmArgs& a, hipStream_t s) {
  switch (a.epi) {
    case MM_GATE: return launch_tiles<T, false, false, MM_GATE>(type, a, s);
    case MM_GATE_BWD: return launch_tiles<T, false, true, MM_GATE_BWD>(type, a, s);
    default:
      if (a.a_rmaj) return launch_tiles<T, true, true, MM_PLAIN>(type, a, s);
      return a.b_rmaj ? launch_tiles<T, false, true, MM_PLAIN>(type, a, s)
                      : launch_tiles<T, false, false, MM_PLAIN>(type, a, s);
  }
}

// Operands whose rows end inside a 16-byte vector (by their extents: what a
// workspace is asked for cannot depend on pointers) are first copied to aligned
// rows where that and the product straight to LDS take less time than the
// product through registers, by the model (10,000 tokens of 1023,
// hidden 4095, g and u then in bf16: forward 430 -> 262 us, backward 1856 -> 653; 3000 rows, 1023
// columns, depth 4095 in 8 bits 49 -> 40; 1024 tokens of 1023, hidden 4095, fp32
// 867 -> 801 forward and backward).
struct Copy {
  const void* src;
  int64_t ld, rows, extent;  // elements
};
int64_t copy_ld(MmType type, int64_t extent) {  // bytes
  return (extent * elem_bytes(type) + 127) / 128 * 128;
}
size_t copy_bytes(MmType type, const Copy& c) { return (size_t)c.rows * (size_t)copy_ld(type, c.extent); }
Copy copy_of_a(const MmArgs& a) { return {a.A, a.lda, a.a_rmaj ? a.K : a.M, a.a_rmaj ? a.M : a.K}; }
Copy copy_of_b(const MmArgs& a) {
  return {a.B, a.ldb, a.b_rmaj ? a.K : is_gate(a.epi) ? 2 * (int64_t)a.N : a.N, a.b_rmaj ? a.N : a.K};
}

double time_of(MmType type, const MmArgs& a, const MmArgs* b, bool dma_a, bool dma_b) {
  const double apart = choose(type, a, dma_a).us + (b ? choose(type, *b, dma_b).us : 0);
  PairPlan p;
  return b && pair_up(type, a, *b, dma_a && dma_b, p) ? p.us : apart;
}

// The operands of a product (or of a pair, whose A is one matrix) that are
// copied, A first; their number.  It depends on the sizes alone.
int copies(MmType type, const MmArgs& a, const MmArgs* b, Copy (&c)[3]) {
  if (a.M < 1 || (b && b->K < 1)) return 0;
  const bool aa = odd_a(type, a) || (b && odd_a(type, *b)), ab = odd_b(type, a), bb = b && odd_b(type, *b);
  if (!aa && !ab && !bb) return 0;
  int n = 0;
  if (aa) c[n++] = copy_of_a(a);
  if (ab) c[n++] = copy_of_b(a);
  if (bb) c[n++] = copy_of_b(*b);
  double us = 5;
  for (int i = 0; i < n; ++i) us += 2.0 * (double)copy_bytes(type, c[i]) / 4e6;
  const double straight = time_of(type, a, b, true, true);
  return us + straight < time_of(type, a, b, !aa && !ab, !aa && !bb) ? n : 0;
}

size_t copies_bytes(MmType type, const Copy* c, int n) {
  size_t bytes = 0;
  for (int i = 0; i < n; ++i) bytes += copy_bytes(type, c[i]);
  return bytes;
}

// Copies the operands that are to be, where the others can go straight to LDS
// as they lie, and points the products to the copies.
hipError_t copy_operands(MmType type, MmArgs& a, MmArgs* b, hipStream_t s) {
  Copy c[3];
  const int n = copies(type, a, b, c);
  if (n == 0) return hipSuccess;
  const size_t bytes = copies_bytes(type, c, n);
  if (a.work_bytes < bytes) return hipErrorInvalidValue;
  const int es = elem_bytes(type);
  MmArgs x = a, y = b ? *b : a;
  CopyArgs k{};
  uint32_t blocks = 0;
  char* dst = reinterpret_cast<char*>(a.work);
  int at = 0;
  auto take = [&](const void*& P, int64_t& ld, int32_t& zero) {
    const int64_t ldd = copy_ld(type, c[at].extent);
    int g = 0;
    while (g < 6 && (16 << g) < ldd) ++g;
    k.src[at] = static_cast<const char*>(c[at].src), k.dst[at] = dst, k.lds[at] = c[at].ld * es, k.ldd[at] = ldd;
    k.width[at] = c[at].extent * es, k.rows[at] = c[at].rows, k.g[at] = g;
    k.blocks[at] = (uint32_t)std::min(cdiv(c[at].rows, 256 >> g), (int64_t)4096);
    blocks += k.blocks[at];
    P = dst, ld = ldd / es, zero = 1;
    dst += copy_bytes(type, c[at++]);
  };
  const bool aa = odd_a(type, a) || (b && odd_a(type, *b));
  if (aa) {
    take(x.A, x.lda, x.a_zero);
    if (b) y.A = x.A, y.lda = x.lda, y.a_zero = 1;
  }
  if (odd_b(type, a)) take(x.B, x.ldb, x.b_zero);
  if (b && odd_b(type, *b)) take(y.B, y.ldb, y.b_zero);
  if (!can_dma(type, x) || (b && !can_dma(type, y))) return hipSuccess;
  for (MmArgs* m : {&x, &y}) m->work = reinterpret_cast<float*>(dst), m->work_bytes = a.work_bytes - bytes;
  hipLaunchKernelGGL(copy_rows_kernel, dim3(blocks), dim3(256), 0, s, k);
  a = x;
  if (b) *b = y;
  return hipGetLastError();
}

hipError_t launch_one(MmType type, const MmArgs& a, hipStream_t s) {
  switch (type) {
    case MM_BF16: return launch_float<__bf16>(type, a, s);
    case MM_FP32: return launch_float<float>(type, a, s);
    default:
      return a.epi == MM_Q8_GATE ? launch_tiles<int8_t, false, false, MM_Q8_GATE>(type, a, s)
                                 : launch_tiles<int8_t, false, false, MM_Q8>(type, a, s);
  }
}

}  // namespace

// (whatever the operands' alignment turns out to be)
size_t mm_workspace(MmType type, const MmArgs& a) {
  Copy c[3];
  const size_t copied = copies_bytes(type, c, copies(type, a, nullptr, c));
  return std::max(copied + partial_bytes(a, choose(type, a, true)), partial_bytes(a, choose(type, a, false)));
}

size_t mm_pair_workspace(MmType type, const MmArgs& a, const MmArgs& b) {
  Copy c[3];
  const size_t copied = copies_bytes(type, c, copies(type, a, &b, c));
  size_t n = 0;
  for (bool dma : {false, true}) {
    size_t part = std::max(partial_bytes(a, choose(type, a, dma)), partial_bytes(b, choose(type, b, dma)));
    PairPlan p;
    if (pair_up(type, a, b, dma, p)) part = std::max(part, pair_bytes(a, b, p));
    n = std::max(n, part + (dma ? copied : 0));
  }
  return n;
}

hipError_t launch_mm(MmType type, const MmArgs& product, hipStream_t s) {
  MmArgs a = product;
  const hipError_t e = copy_operands(type, a, nullptr, s);
  return e == hipSuccess ? launch_one(type, a, s) : e;
}

hipError_t launch_mm_pair(MmType type, const MmArgs& first, const MmArgs& second, hipStream_t s) {
  MmArgs a = first, b = second;
  if (!a.out && !b.out) return hipSuccess;
  const hipError_t copied = copy_operands(type, a, &b, s);
  if (copied != hipSuccess) return copied;
  const bool dma = can_dma(type, a) && can_dma(type, b);
  PairPlan p;
  if (pair_up(type, a, b, dma, p)) {
    if (type == MM_BF16)
      return a.epi == MM_PLAIN ? launch_pair<__bf16, MM_PLAIN>(type, a, b, p, dma, s)
                               : launch_pair<__bf16, MM_GATE_BWD>(type, a, b, p, dma, s);
    return a.epi == MM_PLAIN ? launch_pair<float, MM_PLAIN>(type, a, b, p, dma, s)
                             : launch_pair<float, MM_GATE_BWD>(type, a, b, p, dma, s);
  }
  const hipError_t e = a.out && a.M > 0 ? launch_one(type, a, s) : hipSuccess;
  return e == hipSuccess && b.out ? launch_one(type, b, s) : e;
}

}  // namespace tabpack
