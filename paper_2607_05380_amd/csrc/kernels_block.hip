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
// A K step is 128 bytes of depth (64 bf16, 128 int8, 32 fp32) of 128-row
// regions of 16 KB.  Tiles:
//   small  128 x 128, 4 waves of 64 x 64, two steps in LDS (64 KB), two
//          workgroups per CU.  Operands that do not start rows at 16 bytes or
//          end inside a 16-byte vector, and fp32, pass through registers; the
//          rest go straight to LDS.
//   huge   256 x 256, 8 waves of 128 x 64, two steps in LDS (128 KB), one
//          workgroup per CU (see huge_kernel).
//   thin   up to 64 rows of A, 16 columns, no LDS for operands: each weight
//          byte is read once (see thin_kernel).
// MFMAs: v_mfma_f32_32x32x16_bf16, v_mfma_i32_32x32x32_i8,
// v_mfma_f32_32x32x2_f32, with B as the first operand, so that a lane holds 4
// consecutive columns of one row of C.  Accumulators are fp32 or int32, added
// in a fixed order; a depth split over workgroups is joined in a fixed order
// by a second kernel.
#include <algorithm>

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
// the logistic function; FAST: results that are rounded to bf16 take the
// hardware reciprocal (1 ulp)
template <bool FAST>
__device__ __forceinline__ float logistic(float x) {
  const float d = 1.0f + exp_neg(x);
  return FAST ? __builtin_amdgcn_rcpf(d) : 1.0f / d;
}
constexpr float kSqrtHalf = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;

template <bool FAST>
__device__ __forceinline__ float act_value(int act, float g) {
  if (act == PACK_ACT_SILU) return g * logistic<FAST>(g);
  if (act == PACK_ACT_GELU) return 0.5f * g * (1.0f + erff(g * kSqrtHalf));
  return g > 0.0f ? g : g == g ? 0.0f : g;
}
template <bool FAST>
__device__ __forceinline__ void act_value_grad(int act, float g, float& v, float& d) {
  if (act == PACK_ACT_SILU) {
    const float p = logistic<FAST>(g);
    v = g * p;
    d = p * (1.0f + g * (1.0f - p));
  } else if (act == PACK_ACT_GELU) {
    const float c = 0.5f * (1.0f + erff(g * kSqrtHalf));
    v = g * c;
    d = fmaf(g * kInvSqrt2Pi, __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f), c);
  } else {
    v = g > 0.0f ? g : g == g ? 0.0f : g;
    d = g > 0.0f ? 1.0f : 0.0f;
  }
}

// ---------------------------------------------------------------- epilogues --
// 8 consecutive elements of a row, or the `n` of them that exist; vec: they
// all do and lie at 16 bytes.
__device__ __forceinline__ void load8(const __bf16* p, float* v, int n, bool vec) {
  if (vec) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, u[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float* p, float* v, int n, bool vec) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * i + j] = u[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
  }
}
__device__ __forceinline__ void store8(__bf16* p, const float* v, int n, bool vec) {
  if (vec) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x8*>(p) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (__bf16)v[i];
  }
}
__device__ __forceinline__ void store8(float* p, const float* v, int n, bool vec) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<f32x4*>(p + 4 * i) = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}

// The outputs n .. n + 7 (n < N) of row m from the sums c (gated: gate sums c,
// up sums u), which are consumed.
template <int EPI, typename T>
__device__ __forceinline__ void finish8(const MmArgs& a, int64_t m, int n, float* c, float* u) {
  const int cnt = a.N - n;
  const bool vec = a.vec_out && cnt >= 8;
  constexpr bool FAST = sizeof(T) == 2;
  if constexpr (is_q8(EPI)) {
    const float sx = a.row_scale[m];
    float sw[8], b[8];
    load8(a.col_scale + n, sw, cnt, vec);
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = (float)__builtin_bit_cast(int32_t, c[i]) * (sx * sw[i]);
    if (a.bias) {
      load8(a.bias + n, b, cnt, vec);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] += b[i];
    }
    if constexpr (EPI == MM_Q8_GATE) {
      load8(a.col_scale + a.N + n, sw, cnt, vec);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = (float)__builtin_bit_cast(int32_t, u[i]) * (sx * sw[i]);
      if (a.bias) {
        load8(a.bias + a.N + n, b, cnt, vec);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] += b[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = act_value<false>(a.act, c[i]) * u[i];
    }
    if (a.out_f32)
      store8(static_cast<float*>(a.out) + m * a.ldo + n, c, cnt, vec);
    else
      store8(static_cast<__bf16*>(a.out) + m * a.ldo + n, c, cnt, vec);
  } else if constexpr (EPI == MM_PLAIN) {
    if (a.add) {
      float r[8];
      load8(static_cast<const T*>(a.add) + m * a.ldadd + n, r, cnt, vec);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] += r[i];
    }
    store8(static_cast<T*>(a.out) + m * a.ldo + n, c, cnt, vec);
  } else if constexpr (EPI == MM_GATE) {
    if (a.pre) {
      T* p = static_cast<T*>(a.pre) + m * a.ldpre + n;
      store8(p, c, cnt, vec);
      store8(p + a.N, u, cnt, vec);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = act_value<FAST>(a.act, c[i]) * u[i];
    store8(static_cast<T*>(a.out) + m * a.ldo + n, c, cnt, vec);
  } else {
    static_assert(EPI == MM_GATE_BWD);
    float g[8], w[8], dg[8], du[8];
    const T* p = static_cast<const T*>(a.pre) + m * a.ldpre + n;
    load8(p, g, cnt, vec);
    load8(p + a.N, w, cnt, vec);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v, d;
      act_value_grad<FAST>(a.act, g[i], v, d);
      dg[i] = c[i] * w[i] * d;
      du[i] = c[i] * v;
    }
    T* o = static_cast<T*>(a.out) + m * a.ldo + n;
    store8(o, dg, cnt, vec);
    store8(o + a.N, du, cnt, vec);
  }
}

// Partial sums of a split depth: [split][M][ldp], ldp = N rounded up to 8,
// gated: the up sums in a second such block of columns.
__host__ __device__ __forceinline__ int64_t partial_half(int N) { return ((int64_t)N + 7) / 8 * 8; }
template <int EPI>
__host__ __device__ __forceinline__ int64_t partial_ld(int N) {
  return is_gate(EPI) ? 2 * partial_half(N) : partial_half(N);
}

// One wave's 64 x 64 block of sums acc[i][j] (rows 32 i + lane % 32, columns
// 32 j + ...) to the outputs: through 16 KB of LDS, so that a wave reads and
// writes whole 64-byte (or longer) pieces of rows.  16-byte chunk c of row r
// is stored at c ^ (r & 15).  Gated: columns 0..31 are gate sums, 32..63 the
// up sums of the same outputs.  m0, n0: first row and first output column.
template <int EPI, typename T, typename A16>
__device__ __forceinline__ void store_block(const MmArgs& a, const A16& a00, const A16& a01, const A16& a10,
                                            const A16& a11, char* stage, int m0, int n0, int split, int lane) {
  typedef typename Ty<T>::acc_t acc_t;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const A16& b = i == 0 ? (j == 0 ? a00 : a01) : (j == 0 ? a10 : a11);
      const int row = 32 * i + (lane & 31);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = 8 * j + 2 * q + (lane >> 5);
        typedef acc_t acc4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<acc4*>(stage + row * 256 + ((c ^ (row & 15)) << 4)) =
            acc4{b[4 * q], b[4 * q + 1], b[4 * q + 2], b[4 * q + 3]};
      }
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  constexpr int CH = is_gate(EPI) ? 4 : 8;  // 8-column chunks a row
  constexpr int RP = 64 / CH;               // rows a pass
  const int ch = lane % CH;
  const int n = n0 + 8 * ch;
  if (n < a.N) {
#pragma unroll
    for (int it = 0; it < 64 / RP; ++it) {
      const int row = it * RP + lane / CH;
      const int m = m0 + row;
      if (m < a.M) {
        float c[8], u[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(stage + row * 256 + (((2 * ch + h) ^ (row & 15)) << 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) c[4 * h + e] = v[e];
          if constexpr (is_gate(EPI)) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(stage + row * 256 + (((8 + 2 * ch + h) ^ (row & 15)) << 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) u[4 * h + e] = w[e];
          }
        }
        if (a.splits > 1) {
          float* p = a.work + ((int64_t)split * a.M + m) * partial_ld<EPI>(a.N) + n;
          store8(p, c, 8, true);
          if constexpr (is_gate(EPI)) store8(p + partial_half(a.N), u, 8, true);
        } else {
          finish8<EPI, T>(a, m, n, c, u);
        }
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The sums of a split depth, joined in order of the splits.
template <int EPI, typename T>
__global__ __launch_bounds__(256) void join_kernel(MmArgs a) {
  const int64_t chunks = partial_half(a.N) / 8, total = a.M * chunks;
  const int64_t ldp = partial_ld<EPI>(a.N);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / chunks;
    const int n = (int)(i % chunks) * 8;
    float c[8], u[8], v[8];
    const float* p = a.work + m * ldp + n;
    load8(p, c, 8, true);
    if constexpr (is_gate(EPI)) load8(p + partial_half(a.N), u, 8, true);
    for (int s = 1; s < a.splits; ++s) {
      p += (int64_t)a.M * ldp;
      load8(p, v, 8, true);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (is_q8(EPI))
          c[e] = __builtin_bit_cast(float, __builtin_bit_cast(int32_t, c[e]) + __builtin_bit_cast(int32_t, v[e]));
        else
          c[e] += v[e];
      }
      if constexpr (is_gate(EPI)) {
        load8(p + partial_half(a.N), v, 8, true);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (is_q8(EPI))
            u[e] = __builtin_bit_cast(float, __builtin_bit_cast(int32_t, u[e]) + __builtin_bit_cast(int32_t, v[e]));
          else
            u[e] += v[e];
        }
      }
    }
    finish8<EPI, T>(a, m, n, c, u);
  }
}

// ------------------------------------------------------------------ loaders --
// Straight to LDS (base and rows at 16 bytes, the contiguous extent a multiple
// of 16 bytes): a region is 16 blocks of 1 KB, one load instruction each; wave
// w of NW issues blocks w PER .. w PER + PER - 1.  grow(r): the operand's row
// (rows-contiguous: element) that region row r holds, relative to P, or -1.
// Lanes outside the operand have an offset past the descriptor's range and
// read zeros, so depth past the end adds nothing.
template <int NW, int ES, bool RM>
struct Dma {
  static constexpr int PER = 16 / NW;
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
        const int k = b * 4 + lane / 16;
        const int col = ((((lane % 16) >> 1) ^ rmaj_x<128>(k)) << 4) + (lane & 1) * 8;
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

// Through registers (any alignment and extent): 4 vectors of 16 bytes per
// thread of 256 and region.  rbound: rows-contiguous operands end there.
template <typename T, bool RM>
struct Reg {
  static constexpr int VE = Ty<T>::VE;
  static constexpr int VPR = RM ? 128 / VE : 8;  // vectors per line of the region
  const T* base;
  int64_t ld;
  int64_t row[4];  // operand row (rows-contiguous: element) of the vector, or -1
  int64_t rbound;
  u32x4 v[4];
  template <typename F>
  __device__ __forceinline__ void init(const void* P, int64_t ld_, int64_t rbound_, int tid, F grow) {
    base = static_cast<const T*>(P);
    ld = ld_;
    rbound = rbound_;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = tid + i * 256;
      row[i] = RM ? grow((q % VPR) * VE) : grow(q / VPR);
    }
  }
  __device__ __forceinline__ void load(int64_t k0, int64_t kend, int tid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = tid + i * 256;
      v[i] = u32x4{0, 0, 0, 0};
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
        __builtin_memcpy(&v[i], p, 16);
      } else if (left > 0) {
        T e[VE];
#pragma unroll
        for (int j = 0; j < VE; ++j) e[j] = j < left ? p[j] : (T)0;
        __builtin_memcpy(&v[i], e, 16);
      }
    }
  }
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = tid + i * 256;
      int off;
      if constexpr (!RM)
        off = kmaj16_off<4>(q / VPR, q % VPR);
      else if constexpr (sizeof(T) == 2)
        off = rmaj_off<128>(q / VPR, (q % VPR) * VE);
      else
        off = (q / VPR) * 512 + (q % VPR) * 16;
      *reinterpret_cast<u32x4*>(lds + off) = v[i];
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
template <bool RM>
__device__ __forceinline__ bf16x8 frag_asm(const char* lds, int row, int ks, int lane) {
  if constexpr (RM)
    return frag_tr_asm<128>(lds, row, ks, lane);
  else
    return frag_kmaj_asm<4>(lds, row, ks, lane);
}
// The same as ordinary reads, for regions that were written through registers.
template <typename T, bool RM>
__device__ __forceinline__ bf16x8 frag_reg(const char* lds, int row, int ks, int lane) {
  if constexpr (!RM) {
    return *reinterpret_cast<const bf16x8*>(lds + kmaj16_off<4>(row + (lane & 31), 2 * ks + (lane >> 5)));
  } else if constexpr (sizeof(T) == 2) {
    const int s = lane & 15, g = lane >> 4;
    const int k = 16 * ks + 8 * (g >> 1) + (s >> 2);
    const int col = row + 16 * (g & 1) + 4 * (s & 3);
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + rmaj_off<128>(k, col)));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + rmaj_off<128>(k + 4, col)));
    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
    return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
  } else {  // fp32 [32 depth rows][128]
    f32x4 f;
    const int k = 8 * ks + 4 * (lane >> 5);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = *reinterpret_cast<const float*>(lds + (k + e) * 512 + (row + (lane & 31)) * 4);
    return __builtin_bit_cast(bf16x8, f);
  }
}

// Every LDS read of this wave but the last N is done; the fragments named are
// tied to the wait, so no use of them moves before it.
template <int N>
__device__ __forceinline__ void wait_lds(bf16x8& a, bf16x8& b, bf16x8& c, bf16x8& d) {
  asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(a), "+v"(b), "+v"(c), "+v"(d) : "n"(N < 15 ? N : 15));
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
__device__ __forceinline__ Where where(const MmArgs& a) {
  const uint32_t per = (uint32_t)a.tiles_m * a.tiles_n;
  Where w;
  w.split = blockIdx.x / per;
  const uint32_t b = blockIdx.x % per, q = per / 8, r = per % 8, x = b % 8;
  const uint32_t t = x * q + (x < r ? x : r) + b / 8;
  const uint32_t band = t / (4 * a.tiles_n), in = t % (4 * a.tiles_n);
  const uint32_t h = min(4u, (uint32_t)a.tiles_m - 4 * band);
  w.tm = 4 * band + in % h;
  w.tn = in / h;
  return w;
}

// ------------------------------------------------------------- small tiles --
template <typename T, bool RA, bool RB, int EPI, bool DMA>
__global__ __launch_bounds__(256, 2) void small_kernel(MmArgs a) {
  constexpr int ES = sizeof(T), KE = kStep / ES;
  __shared__ __attribute__((aligned(16))) char smem[4 * kRegion];
  typedef typename Ty<T>::acc16 acc16;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const Where w = where(a);
  const int m0 = w.tm * 128, n0 = w.tn * (is_gate(EPI) ? 64 : 128);
  const int64_t kbeg = (int64_t)w.split * a.steps_per_split * KE;
  const int64_t kend = min((int64_t)a.K, kbeg + (int64_t)a.steps_per_split * KE);
  const int nk = (int)((kend - kbeg + KE - 1) / KE);
  auto grow_a = [&](int r) -> int64_t { return m0 + r < a.M ? r : -1; };
  // region row wn 64 + j 32 + x: plain column n0 + that; gated: gate (j = 0) or
  // up (j = 1) row of output n0 + wn 32 + x
  auto grow_b = [&](int r) -> int64_t {
    if constexpr (!is_gate(EPI)) return n0 + r < a.N ? r : -1;
    const int x = (r >> 6) * 32 + (r & 31);
    return n0 + x < a.N ? x + ((r >> 5) & 1 ? (int64_t)a.N : 0) : -1;
  };
  const T* A = static_cast<const T*>(a.A) + (RA ? (int64_t)m0 : m0 * a.lda);
  const T* B = static_cast<const T*>(a.B) + (RB ? (int64_t)n0 : n0 * a.ldb);
  acc16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) clear(acc[i][j]);
  if constexpr (DMA) {
    Dma<4, ES, RA> la;
    Dma<4, ES, RB> lb;
    la.init(A, a.lda, wave, lane, grow_a);
    lb.init(B, a.ldb, wave, lane, grow_b);
    auto issue = [&](char* st, int64_t k0) {
#pragma unroll
      for (int p = 0; p < 4; ++p) la.issue(st, k0, kend, p);
#pragma unroll
      for (int p = 0; p < 4; ++p) lb.issue(st + kRegion, k0, kend, p);
    };
    constexpr int NRD = (RA ? 4 : 2) + (RB ? 4 : 2);  // LDS reads per MFMA step
    issue(smem, kbeg);
#pragma unroll 1
    for (int kt = 0; kt < nk; ++kt) {
      char* const cur = smem + (kt & 1) * 2 * kRegion;
      wait_vm<0, true>();
      bar();  // this step has landed, and every wave is done with the last one
      if (kt + 1 < nk) issue(smem + ((kt + 1) & 1) * 2 * kRegion, kbeg + (int64_t)(kt + 1) * KE);
      bf16x8 fa[4][2], fb[4][2];
      auto rd = [&](int ks) {
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[ks][i] = frag_asm<RA>(cur, wm * 64 + i * 32, ks, lane);
#pragma unroll
        for (int j = 0; j < 2; ++j) fb[ks][j] = frag_asm<RB>(cur + kRegion, wn * 64 + j * 32, ks, lane);
      };
      rd(0);
      rd(1);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        if (ks + 2 < 4) rd(ks + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (ks < 2)
          wait_lds<2 * NRD>(fa[ks][0], fa[ks][1], fb[ks][0], fb[ks][1]);
        else if (ks == 2)
          wait_lds<NRD>(fa[ks][0], fa[ks][1], fb[ks][0], fb[ks][1]);
        else
          wait_lds<0>(fa[ks][0], fa[ks][1], fb[ks][0], fb[ks][1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) mma(fb[ks][j], fa[ks][i], acc[i][j], T());
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    Reg<T, RA> la;
    Reg<T, RB> lb;
    la.init(A, a.lda, a.M - m0, tid, grow_a);
    lb.init(B, a.ldb, a.N - n0, tid, grow_b);
    la.load(kbeg, kend, tid);
    lb.load(kbeg, kend, tid);
#pragma unroll 1
    for (int kt = 0; kt < nk; ++kt) {
      char* const cur = smem + (kt & 1) * 2 * kRegion;
      la.store(cur, tid);
      lb.store(cur + kRegion, tid);
      __syncthreads();  // the other stage was read before the barrier of the step before this one's stores
      if (kt + 1 < nk) {
        la.load(kbeg + (int64_t)(kt + 1) * KE, kend, tid);
        lb.load(kbeg + (int64_t)(kt + 1) * KE, kend, tid);
      }
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        bf16x8 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[i] = frag_reg<T, RA>(cur, wm * 64 + i * 32, ks, lane);
#pragma unroll
        for (int j = 0; j < 2; ++j) fb[j] = frag_reg<T, RB>(cur + kRegion, wn * 64 + j * 32, ks, lane);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) mma(fb[j], fa[i], acc[i][j], T());
      }
    }
  }
  wait_vm<0, true>();
  bar();  // the sums are staged in the operand regions
  store_block<EPI, T>(a, acc[0][0], acc[0][1], acc[1][0], acc[1][1], smem + wave * 16384, m0 + wm * 64,
                      n0 + wn * (is_gate(EPI) ? 32 : 64), w.split, lane);
}

// ------------------------------------------------------------------- host --
struct Plan {
  int tm, tn, splits, steps;
};

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

int elem_bytes(MmType t) { return t == MM_BF16 ? 2 : t == MM_FP32 ? 4 : 1; }

// Tiles of a product and how many workgroups share each tile's depth: as many
// as fill the chip's 512 small-tile places, at least 8 steps each.
Plan plan_small(MmType type, const MmArgs& a) {
  Plan p;
  p.tm = (int)cdiv(a.M, 128);
  p.tn = (int)cdiv(a.N, is_gate(a.epi) ? 64 : 128);
  const int64_t steps = a.K > 0 ? cdiv((int64_t)a.K * elem_bytes(type), kStep) : 1;
  const int64_t tiles = std::max((int64_t)p.tm * p.tn, (int64_t)1);  // (no rows: a workspace query)
  int64_t s = tiles >= 256 ? 1 : 512 / tiles;
  s = s < steps / 8 ? s : steps / 8;
  if (s < 1) s = 1;
  p.steps = (int)cdiv(steps, s);
  p.splits = (int)cdiv(steps, p.steps);
  return p;
}

size_t partial_bytes(const MmArgs& a, const Plan& p) {
  if (p.splits < 2) return 0;
  return (size_t)p.splits * (size_t)a.M * (size_t)partial_half(a.N) * (is_gate(a.epi) ? 8 : 4);
}

bool rows16(const void* p, int64_t ld, int es, int64_t extent) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0 && extent * es % 16 == 0;
}

// Whether both operands can go straight to LDS: rows at 16 bytes, whole 16-byte
// vectors, and tile-relative offsets below 2 GiB.
bool can_dma(MmType type, const MmArgs& a) {
  if (type == MM_FP32) return false;
  const int es = elem_bytes(type);
  if (!rows16(a.A, a.lda, es, a.a_rmaj ? a.M : a.K) || !rows16(a.B, a.ldb, es, a.b_rmaj ? a.N : a.K)) return false;
  const int64_t lim = (int64_t)1 << 31;
  const int64_t brows = is_gate(a.epi) ? (int64_t)a.N + 256 : 256;
  return a.lda * es * 256 < lim && a.ldb * es * brows < lim && (int64_t)a.K * es < lim / 2;
}

template <typename T, bool RA, bool RB, int EPI>
hipError_t launch_tiles(MmType type, MmArgs a, hipStream_t s) {
  const Plan p = plan_small(type, a);
  a.tiles_m = p.tm, a.tiles_n = p.tn, a.splits = p.splits, a.steps_per_split = p.steps;
  const int64_t blocks = (int64_t)p.tm * p.tn * p.splits;
  if (blocks > (1 << 23)) return hipErrorInvalidConfiguration;  // a launch is limited to 2^32 threads
  const dim3 grid((uint32_t)blocks);
  bool dma = false;
  if constexpr (sizeof(T) != 4) {
    dma = can_dma(type, a);
    if (dma) hipLaunchKernelGGL((small_kernel<T, RA, RB, EPI, true>), grid, dim3(256), 0, s, a);
  }
  if (!dma) hipLaunchKernelGGL((small_kernel<T, RA, RB, EPI, false>), grid, dim3(256), 0, s, a);
  if (p.splits > 1) {
    const int64_t n = cdiv((int64_t)a.M * (partial_half(a.N) / 8), 256);
    hipLaunchKernelGGL((join_kernel<EPI, T>), dim3((uint32_t)(n < 4096 ? n : 4096)), dim3(256), 0, s, a);
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

}  // namespace

size_t mm_workspace(MmType type, const MmArgs& a) { return partial_bytes(a, plan_small(type, a)); }

hipError_t launch_mm(MmType type, const MmArgs& args, hipStream_t s) {
  MmArgs a = args;
  // outputs, added and saved matrices in 16-byte pieces where all allow it
  const int es = type == MM_BF16 || (type == MM_I8 && !a.out_f32) ? 2 : 4;
  auto ok = [&](const void* p, int64_t ld) { return !p || rows16(p, ld, es, a.N); };
  auto okv = [&](const float* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  a.vec_out = a.N % 8 == 0 && ok(a.out, a.ldo) && ok(a.add, a.ldadd) && ok(a.pre, a.ldpre) && okv(a.col_scale) &&
              okv(a.bias);
  switch (type) {
    case MM_BF16: return launch_float<__bf16>(type, a, s);
    case MM_FP32: return launch_float<float>(type, a, s);
    default:
      return a.epi == MM_Q8_GATE ? launch_tiles<int8_t, false, false, MM_Q8_GATE>(type, a, s)
                                 : launch_tiles<int8_t, false, false, MM_Q8>(type, a, s);
  }
}

}  // namespace tabpack
