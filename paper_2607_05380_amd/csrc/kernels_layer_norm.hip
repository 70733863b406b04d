// Layer norm of a student network on gfx950: v = x + residual less its row mean,
// divided by its deviation, and the gradients of x, the weight and the bias.
//
// A row is read once into the registers of the G threads that own it (4 to
// 1024, EPT elements each), so the mean, the mean square about it and the
// output come from one read, and the bytes of one read and one write bound the
// forward pass and the row's gradient.  The deviation is that of the differences
// v - mean, not a difference of mean squares, which would lose rows whose mean
// is large beside it; and the differences' own mean, what rounding left in the
// first one, is taken out of them.
//
// Measured: 65,536 x 1024 bf16 with residual 91 us forward (5.9 TB/s of reads and
// writes), 112 backward (4.8) and 5 for the sums of the weight and bias; 4095 x
// 1023 fp32, rows at 4 bytes, 13, 17 and 5 us (two rows a thread group at least:
// with one the partial sums take 3 us more, with four the rows 2).
// Rows past 8192 columns take 1024 threads of 128 registers: 4096 x 16,384 bf16 122
// and 210 us (its bytes 104 and 78); past 16,384 in fp32 they spill, 23 registers
// forward and 45 backward (2048 x 32,768 255 and 422 us, 207 and 156), and the
// backward pass reads v three times and dy twice.
#include "ops_internal.h"
#include "row_tiles.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

// The sums over a row's G threads of N values, behind one barrier (red: N times 16 floats, as reduce_row's).
template <int G, int N>
__device__ __forceinline__ void reduce_rows(float (&v)[N], float (*red)[16], int tid) {
#pragma unroll
  for (int m = (G < 64 ? G : 64) / 2; m >= 1; m >>= 1)
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] += __shfl_xor(v[q], m, 64);
  if constexpr (G > 64) {
    if ((tid & 63) == 0)
#pragma unroll
      for (int q = 0; q < N; ++q) red[q][tid >> 6] = v[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < N; ++q) {
      if constexpr (G == 1024) {  // (16 words of each sum would not fit its registers)
        v[q] = red[q][tid & 15];
#pragma unroll
        for (int m = 8; m >= 1; m >>= 1) v[q] += __shfl_xor(v[q], m, 64);
      } else {
        v[q] = red[q][0];
#pragma unroll
        for (int w = 1; w < G / 64; ++w) v[q] += red[q][w];
      }
    }
  }
}

// ---------------------------------------------------------------- forward --
// mu = mean v, rho = (mean (v - mu)^2 + eps)^(-1/2), y = (v - mu) rho w + b.
// The sum's rounding leaves the mean m off by some 2^-24 |m|, which shows where
// the deviation is small beside it (a mean of 1e5 and a deviation of 1: y off by
// 1e-2).  So mu = m + e with e = mean (v - m), and mean (v - mu)^2 =
// mean (v - m)^2 - e^2: both sums stand behind one barrier.  Where e^2 is no
// longer small beside the mean square that difference loses digits, and the row
// goes through its sums again about m + e rounded, whose e is at most half a
// step of the mean; values lie on steps no smaller than that unless the deviation is
// of the mean's size, so then e^2 is at most the variance.  (Against one sum of the
// differences' squares, in turn on one card: 65,536 x 1024 bf16 94 us both ways,
// 500,000 x 64 67 -> 71.)
// Where a sum or a square overflows (values past 1.8e19) the row goes on 2^-80
// times smaller, and where squares leave fp32's range at its lower end (with an
// eps there too) 2^80 times larger, neither of which changes y.  A row of equal
// values has no differences, whatever its scale, and eps alone makes its rho.  A
// row that holds an infinity or NaN is NaN throughout.
template <typename T, int G, int EPT>
__global__ __launch_bounds__(G > 256 ? G : 256) void layer_norm_kernel(LayerNormArgs a) {
  constexpr int VE = kVec<T>, NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE;
  __shared__ float red[2][7][16];
  const int tid = threadIdx.x, t = tid % G;
  static_assert(G <= 64 || RPB == 1, "a row's barriers are the block's");
  int turn = 0;  // rows take turns with two sets of LDS words: a row's barriers lie between their uses
  for (int64_t row = (int64_t)blockIdx.x * RPB + tid / G; row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
    Vec<T> xs[NV], rs[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      xs[i].load(x + c, a.cols - c);
      if (r) rs[i].load(r + c, a.cols - c);
    }
    float v[EPT], total = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      xs[i].get(v + i * VE);
      if (r) {
        float u[VE];
        rs[i].get(u);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[i * VE + e] += u[e];
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) total += v[i * VE + e];
    }
    if (a.sum) {
      T* s = static_cast<T*>(a.sum) + row * a.lds;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VE;
        store_vec(s + c, v + i * VE, a.cols - c);
      }
    }
    // the differences' sum and that of their squares
    float s1, s2;
    auto about = [&](float m, int at) {
      s1 = s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float d = (i * G + t) * VE + e < a.cols ? v[i * VE + e] - m : 0.0f;
          s1 += d;
          s2 = fmaf(d, d, s2);
        }
      float both[2] = {s1, s2};
      reduce_rows<G>(both, &red[turn][at], tid);
      s1 = both[0], s2 = both[1];
    };
    const float n = (float)a.cols;
    float shift = reduce_row<G, OpAdd>(total, red[turn][0], tid) / n;
    about(shift, 1);
    float e1 = s1 / n, by = 1.0f;
    const bool over = !(s2 < __builtin_inff()), under = s2 + n * a.eps < 0x1p-100f && fabsf(shift) < 1.0f;
    if (over || under || e1 * s1 > 0x1p-12f * (s2 + n * a.eps)) {  // (the same for all threads of the row)
      if (over || under) {
        by = over ? 0x1p-80f : 0x1p80f;
        total = 0.0f;
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
          v[e] *= by;
          total += v[e];
        }
        shift = reduce_row<G, OpAdd>(total, red[turn][3], tid) / n;
        s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VE; ++e) s1 += (i * G + t) * VE + e < a.cols ? v[i * VE + e] - shift : 0.0f;
        e1 = reduce_row<G, OpAdd>(s1, red[turn][4], tid) / n;
      }
      shift += e1;
      about(shift, 5);
      e1 = s1 / n;
    }
    float var = s2 / n - e1 * e1;
    var = var < 0.0f ? 0.0f : var;  // (NaN stays)
    const float rho = 1.0f / sqrtf(s2 == 0.0f ? a.eps : var + a.eps * by * by), rstd = s2 == 0.0f ? rho : rho * by;
    float mean = shift + e1;
    if (by > 1.0f) mean *= 0x1p-80f;
    if (by < 1.0f) {
      // (a mean of the largest values may round past them)
      const float m = mean * 0x1p80f;
      mean = fabsf(m) == __builtin_inff() && fabsf(mean) < 0x1p49f ? copysignf(3.402823466e38f, m) : m;
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    T* o = static_cast<T*>(a.out) + row * a.ldo;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      float w[VE], b[VE];
      load_weight<VE>(a.weight + c, w, a.cols - c);
      if (a.bias) {
        load_weight<VE>(a.bias + c, b, a.cols - c);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) b[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) w[e] = fmaf((v[i * VE + e] - shift - e1) * rho, w[e], b[e]);
      store_vec(o + c, w, a.cols - c);
    }
  }
}

// --------------------------------------------------------------- backward --
// With n = (v - mean) rstd, g = w dy and D = cols:
//   dx = rstd (g - sum(g) / D - n sum(g n) / D) + dsum,
//   dweight = sum over the rows of dy n,  dbias = sum over the rows of dy.
// (n is formed as (v / 2 - mean / 2) 2 rstd, whose difference cannot overflow.)
// In fp32, where v is stored as the norm took it, n less its own row mean h, what
// the mean's rounding left in it, stands for n: 2^-24 |mean| rstd, 0.03 for rows of
// 1e6 +- 1; sum(g (n - h)) = sum(g n) - h sum(g).  (In bf16 v's own rounding counts
// for more.)  65,536 x 1024 fp32 187 us before, 189 with it, 8192 x 8192 232 and 245.
// A block walks over rows (gridDim apart) and keeps the columns' two sums in
// registers; they go to one row of `partial`, and a second kernel adds these up
// in order: no atomics, so the result does not change between runs.  SUMS false:
// rows past 16,384 columns, whose sums leave the registers no room; a kernel of
// columns reads dy and v again for them.
template <typename T, int G, int EPT, bool SUMS>
__global__ __launch_bounds__(G > 256 ? G : 256) void layer_norm_bwd_kernel(LayerNormBwdArgs a) {
  constexpr int VE = kVec<T>, NT = G > 256 ? G : 256, RPB = NT / G, NV = EPT / VE, NS = SUMS ? EPT : 1;
  constexpr bool LATE = G > 256;  // dsum is read behind the sums (the registers of 1024 threads do not hold it)
  constexpr bool OFF = sizeof(T) == 4;
  __shared__ float red[2][OFF ? 3 : 2][16];
  __shared__ float cols[RPB > 1 ? 2 * G * EPT : 1];
  const int tid = threadIdx.x, t = tid % G, rg = tid / G;
  float dw[NS], db[NS];
#pragma unroll
  for (int e = 0; e < NS; ++e) dw[e] = db[e] = 0.0f;
  int turn = 0;  // (as in layer_norm_kernel)
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
      if (!LATE && ds)
        os[i].load(ds + c, a.cols - c);
      else
        os[i].raw = u32x4{0, 0, 0, 0};
    }
    const float rho = a.rstd[row], half = -0.5f * a.mean[row], twice = 2.0f * rho;
    float sg = 0.0f, sgn = 0.0f, sn = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      float w[VE], v[VE], g[VE];
      load_weight<VE>(a.weight + c, w, a.cols - c);
      vs[i].get(v);
      gs[i].get(g);
#pragma unroll
      for (int e = 0; e < VE; ++e) {  // (behind the row's end g and w are 0)
        const float n = fmaf(v[e], 0.5f, half) * twice;
        if constexpr (SUMS) {
          if constexpr (!OFF) dw[i * VE + e] = fmaf(g[e], n, dw[i * VE + e]);
          db[i * VE + e] += g[e];
        }
        if constexpr (OFF) sn += c + e < a.cols ? n : 0.0f;
        g[e] *= w[e];
        sg += g[e];
        sgn = fmaf(g[e], n, sgn);
      }
    }
    const float n = (float)a.cols;
    float sums[OFF ? 3 : 2] = {sg, sgn};
    if constexpr (OFF) sums[2] = sn;
    reduce_rows<G>(sums, red[turn], tid);
    const float c1 = sums[0] / n, off = OFF ? sums[OFF ? 2 : 0] / n : 0.0f, c2 = fmaf(-off, c1, sums[1] / n);
    T* dx = static_cast<T*>(a.dx) + row * a.ldx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VE;
      float w[VE], v[VE], g[VE], o[VE];
      load_weight<VE>(a.weight + c, w, a.cols - c);
      vs[i].get(v);
      gs[i].get(g);
      if (LATE && ds) os[i].load(ds + c, a.cols - c);
      os[i].get(o);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float nn = fmaf(v[e], 0.5f, half) * twice - off;
        if constexpr (SUMS && OFF) dw[i * VE + e] = fmaf(g[e], nn, dw[i * VE + e]);
        o[e] = fmaf(rho, (g[e] * w[e] - c1) - nn * c2, o[e]);
      }
      store_vec(dx + c, o, a.cols - c);
    }
  }
  if constexpr (SUMS) {
    float* const out = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (RPB > 1) {  // the block's sums: its row groups one after the other
      for (int r = 0; r < RPB; ++r) {
        if (rg == r) {
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              const int c = (i * G + t) * VE + e;
              cols[c] = (r == 0 ? 0.0f : cols[c]) + dw[i * VE + e];
              cols[G * EPT + c] = (r == 0 ? 0.0f : cols[G * EPT + c]) + db[i * VE + e];
            }
        }
        __syncthreads();
      }
      for (int c = tid; c < a.cols; c += NT) {
        out[c] = cols[c];
        out[a.cols + c] = cols[G * EPT + c];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int c = (i * G + t) * VE + e;
          if (c < a.cols) {
            out[c] = dw[i * VE + e];
            out[a.cols + c] = db[i * VE + e];
          }
        }
    }
  }
}

// The row means of wide rows' n (fp32).
__global__ __launch_bounds__(1024) void layer_norm_off_kernel(LayerNormBwdArgs a) {
  __shared__ float red[2][16];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const float* const s = static_cast<const float*>(a.sum) + row * a.lds;
    const float half = -0.5f * a.mean[row], twice = 2.0f * a.rstd[row];
    float sn = 0.0f;
#pragma unroll 8
    for (int c = threadIdx.x * 4; c < a.cols; c += 4096) {
      Vec<float> vs;
      float v[4];
      vs.load(s + c, a.cols - c);
      vs.get(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) sn += c + e < a.cols ? fmaf(v[e], 0.5f, half) * twice : 0.0f;
    }
    sn = reduce_row<1024, OpAdd>(sn, red[turn], threadIdx.x);
    if (threadIdx.x == 0) a.off[row] = sn / (float)a.cols;
  }
}

// The sums of wide rows: a block takes 64 vectors of columns and every gridDim.y-th
// group of 4 rows.
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_cols_kernel(LayerNormBwdArgs a) {
  constexpr int VE = kVec<T>;
  __shared__ float part[2][4][64 * VE];
  const int lane = threadIdx.x & 63, rg = threadIdx.x >> 6;
  const int c = (blockIdx.x * 64 + lane) * VE;
  float dw[VE], db[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) dw[e] = db[e] = 0.0f;
  if (c < a.cols) {
#pragma unroll 4
    for (int64_t row = (int64_t)blockIdx.y * 4 + rg; row < a.rows; row += (int64_t)gridDim.y * 4) {
      Vec<T> vs, gs;
      vs.load(static_cast<const T*>(a.sum) + row * a.lds + c, a.cols - c);
      gs.load(static_cast<const T*>(a.dy) + row * a.ldy + c, a.cols - c);
      const float half = -0.5f * a.mean[row], twice = 2.0f * a.rstd[row];
      const float off = sizeof(T) == 4 ? a.off[row] : 0.0f;
      float v[VE], g[VE];
      vs.get(v);
      gs.get(g);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        dw[e] = fmaf(g[e], fmaf(v[e], 0.5f, half) * twice - off, dw[e]);
        db[e] += g[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < VE; ++e) part[0][rg][lane * VE + e] = dw[e], part[1][rg][lane * VE + e] = db[e];
  __syncthreads();
  float* const out = a.partial + (int64_t)blockIdx.y * 2 * a.cols;
  for (int i = threadIdx.x; i < 64 * VE; i += 256) {
    const int at = blockIdx.x * 64 * VE + i;
    if (at < a.cols) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        out[h * a.cols + at] = ((part[h][0][i] + part[h][1][i]) + part[h][2][i]) + part[h][3][i];
    }
  }
}

// dweight and dbias from the blocks' partial sums: 16 columns and 64 row
// streams a block
__global__ __launch_bounds__(1024) void layer_norm_sums_kernel(const float* partial, int nblk, int cols, float* dw,
                                                               float* db) {
  __shared__ float part[64][17];
  const int i = threadIdx.x % 16, c = blockIdx.x * 16 + i, r = threadIdx.x / 16;
  float s = 0.0f;
  if (c < 2 * cols) {
#pragma unroll 8
    for (int b = r; b < nblk; b += 64) s += partial[(int64_t)b * 2 * cols + c];
  }
  part[r][i] = s;
  __syncthreads();
  if (r == 0 && c < 2 * cols) {
    for (int q = 1; q < 64; ++q) s += part[q][i];
    if (c < cols)
      dw[c] = s;
    else if (db)
      db[c - cols] = s;
  }
}

template <typename T>
hipError_t forward_t(const LayerNormArgs& a, hipStream_t s) {
#define TABPACK_LN(G, EPT)                                                                             \
  if (a.cols <= G * EPT) {                                                                             \
    constexpr int RPB = G > 256 ? 1 : 256 / G;                                                         \
    hipLaunchKernelGGL((layer_norm_kernel<T, G, EPT>), dim3(row_blocks(a.rows, RPB)),                  \
                       dim3(G > 256 ? G : 256), 0, s, a);                                              \
    return hipGetLastError();                                                                          \
  }
  TABPACK_LN(4, 8)
  TABPACK_LN(16, 8)
  TABPACK_LN(64, 8)
  TABPACK_LN(64, 16)
  TABPACK_LN(64, 32)
  TABPACK_LN(256, 16)
  TABPACK_LN(256, 32)
  TABPACK_LN(1024, 16)
  TABPACK_LN(1024, 32)
#undef TABPACK_LN
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t backward_t(const LayerNormBwdArgs& a, hipStream_t s) {
  const int nblk = layer_norm_bwd_blocks(a.rows, a.cols);
  const dim3 sums((2 * a.cols + 15) / 16);
#define TABPACK_LN_BWD(G, EPT)                                                                                \
  if (a.cols <= G * EPT) {                                                                                    \
    hipLaunchKernelGGL((layer_norm_bwd_kernel<T, G, EPT, true>), dim3(nblk), dim3(G > 256 ? G : 256), 0, s, a);     \
    hipLaunchKernelGGL(layer_norm_sums_kernel, sums, dim3(1024), 0, s, a.partial, nblk, a.cols, a.dweight, a.dbias); \
    return hipGetLastError();                                                                                 \
  }
  TABPACK_LN_BWD(4, 8)
  TABPACK_LN_BWD(16, 8)
  TABPACK_LN_BWD(64, 8)
  TABPACK_LN_BWD(64, 16)
  TABPACK_LN_BWD(64, 32)
  TABPACK_LN_BWD(256, 16)
  TABPACK_LN_BWD(256, 32)
  TABPACK_LN_BWD(1024, 16)
#undef TABPACK_LN_BWD
  if (a.cols > kRowMaxCols) return hipErrorInvalidValue;
  // the sums first: dx may take dy's place
  const int columns = 64 * kVec<T>;
  if (sizeof(T) == 4 && a.rows > 0)
    hipLaunchKernelGGL(layer_norm_off_kernel, dim3(row_blocks(a.rows, 1)), dim3(1024), 0, s, a);
  hipLaunchKernelGGL((layer_norm_cols_kernel<T>), dim3((a.cols + columns - 1) / columns, nblk), dim3(256), 0, s, a);
  hipLaunchKernelGGL(layer_norm_sums_kernel, sums, dim3(1024), 0, s, a.partial, nblk, a.cols, a.dweight, a.dbias);
  if (a.rows > 0)
    hipLaunchKernelGGL((layer_norm_bwd_kernel<T, 1024, 32, false>), dim3(row_blocks(a.rows, 1)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Rows of partial sums: up to 16,384 columns those of the root-mean-square norm's
// backward pass over half as many rows (the sums are twice as many, see above),
// past them 64 groups of rows, of 32 rows at least, for each block of columns.
int layer_norm_bwd_blocks(int64_t rows, int32_t cols) {
  if (cols <= 16384) return norm_bwd_blocks((rows + 1) / 2, cols);
  const int64_t want = (rows + 31) / 32;
  return (int)(want < 64 ? (want > 0 ? want : 1) : 64);
}

// Rows past 16,384 columns: a float each.
int64_t layer_norm_bwd_offs(int64_t rows, int32_t cols) { return cols <= 16384 ? 0 : rows; }

hipError_t launch_layer_norm(int prec, const LayerNormArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? forward_t<__bf16>(a, s) : forward_t<float>(a, s);
}
hipError_t launch_layer_norm_bwd(int prec, const LayerNormBwdArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? backward_t<__bf16>(a, s) : backward_t<float>(a, s);
}

}  // namespace tabpack
