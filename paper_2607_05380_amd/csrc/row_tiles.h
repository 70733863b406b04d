// What the row kernels share (kernels_rows.hip, kernels_layer_norm.hip,
// kernels_embed_table.hip, kernels_dropout.hip, kernels_quant.hip): vectors of
// 16 bytes at any alignment of the element, reductions over the threads of a row,
// blocks of a launch over rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

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

// blocks of a launch over rows, rpb of them a block (a launch is limited to
// 2^32 threads; a block goes on with the rows past the grid)
uint32_t row_blocks(int64_t rows, int rpb) {
  const int64_t n = (rows + rpb - 1) / rpb;
  return (uint32_t)(n < (1 << 20) ? n : 1 << 20);
}

}  // namespace
}  // namespace tabpack
