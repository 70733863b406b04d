// 8-bit floating point codes (e4m3: 3 bits of mantissa, up to 448) with a scale
// for each block: of 128 columns of a row (activations), or of 128 x 128 of a
// matrix (weights).  q = e4m3(x 448 / max|x|), rounded to the nearest code (ties
// to the even one), scale = max|x| / 448 over the block.
//
// Activations' scales lie [blocks, rows]: the product reads those of a step's
// rows together.  One read and one write bound both kernels: rows of 20,011 x
// 4096 bf16 in 37-39 us (6.3-6.6 TB/s), 2048 x 2048 in 4; tiles of 20,011 x 4096
// in 39 us, of 8192 x 8192 bf16 in 32 (6.3 TB/s), fp32 in 60 (5.6).
#include <algorithm>

#include "ops_internal.h"
#include "row_tiles.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

constexpr int kBlock = PACK_F8_BLOCK;

// 448 / a, 0 where a is 0 or so small that the quotient overflows (a block of
// such values has codes 0 and scale 0)
__device__ __forceinline__ float f8_factor(float a) {
  const float f = 448.0f / a;
  return a > 0.0f && f < __builtin_inff() ? f : 0.0f;
}

// 8 elements as floats: the first n at p, the others 0
template <typename T>
struct Eight {
  Vec<T> raw[8 / kVec<T>];
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int i = 0; i < 8 / kVec<T>; ++i) raw[i].load(p + i * kVec<T>, n - i * kVec<T>);
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int i = 0; i < 8 / kVec<T>; ++i) raw[i].get(v + i * kVec<T>);
  }
};

// The first n of 8 codes of v f.
__device__ __forceinline__ void store_f8(uint8_t* p, const float* v, float f, int n) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float* x = v + 4 * h;
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, c, true);
  }
  if (n >= 8) {
    *reinterpret_cast<u32x2_any*>(p) = u32x2{w[0], w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// The factor of a block whose largest magnitude is m, and its scale: codes of a
// block that holds an infinity or NaN are 0 (their values times 0 would not be:
// `finite` says so) and its scale NaN.
struct BlockScale {
  float factor, scale;
  bool finite;
  __device__ __forceinline__ explicit BlockScale(float m) {
    finite = m < __builtin_inff();
    factor = finite ? f8_factor(m) : 0.0f;
    scale = !finite ? __builtin_nanf("") : factor == 0.0f ? 0.0f : m / 448.0f;
  }
};

// A workgroup: 16 rows of one block of columns, 16 threads a row.  first: the
// launch's first workgroup of all (a launch is limited to 2^32 threads; a loop over
// them in the kernel instead cost 20,011 x 4096 bf16 4%).
template <typename T>
__global__ __launch_bounds__(256) void row_codes_kernel(BlockCodeArgs a, uint32_t blocks, uint32_t first) {
  const int t = threadIdx.x % 16;
  const uint32_t unit = first + blockIdx.x, b = unit % blocks;
  const int64_t row = (int64_t)(unit / blocks) * 16 + threadIdx.x / 16;
  if (row >= a.rows) return;
  const int c = (int)b * kBlock + t * 8, n = a.cols - c;
  Eight<T> x;
  float v[8], m = 0.0f;
  x.load(static_cast<const T*>(a.x) + row * a.ldx + c, n);
  x.get(v);
#pragma unroll
  for (int i = 0; i < 8; ++i) m = OpMaxMag::op(m, fabsf(v[i]));
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) m = OpMaxMag::op(m, __shfl_xor(m, d, 64));
  const BlockScale s(m);
  if (!s.finite)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
  if (n > 0) store_f8(a.q + row * a.ldq + c, v, s.factor, n);
  if (t == 0) a.scale[(int64_t)b * a.rows + row] = s.scale;
}

// A workgroup: one tile, 16 threads a row and 8 rows a thread.
template <typename T>
__global__ __launch_bounds__(256) void tile_codes_kernel(BlockCodeArgs a, uint32_t blocks, uint32_t tiles,
                                                         uint32_t first) {
  __shared__ float red[4];
  const int t = threadIdx.x % 16, r = threadIdx.x / 16;
  const uint32_t unit = first + blockIdx.x, b = unit % blocks, tile = unit / blocks;  // (tile: of all parts)
  const int64_t part = tile / tiles, row0 = (int64_t)(tile % tiles) * kBlock + r;
  const int c = (int)b * kBlock + t * 8, n = a.cols - c;
  const T* x = static_cast<const T*>(a.x) + part * a.rows * a.ldx + c;
  Eight<T> e[8];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    // (rows past the end read row 0 of the part, of which no element counts)
    e[i].load(x + (row < a.rows ? row : 0) * a.ldx, row < a.rows ? n : 0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    e[i].get(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = OpMaxMag::op(m, fabsf(v[j]));
  }
  m = reduce_row<256, OpMaxMag>(m, red, threadIdx.x);
  const BlockScale s(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    float v[8];
    e[i].get(v);
    if (!s.finite)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    if (row < a.rows && n > 0) store_f8(a.q + (part * a.rows + row) * a.ldq + c, v, s.factor, n);
  }
  if (threadIdx.x == 0) a.scale[(int64_t)tile * blocks + b] = s.scale;
}

}  // namespace

hipError_t launch_block_codes(int prec, bool tile, const BlockCodeArgs& a, hipStream_t s) {
  const int64_t blocks = (a.cols + kBlock - 1) / kBlock, tiles = (a.rows + kBlock - 1) / kBlock;
  const int64_t n = tile ? a.parts * tiles * blocks : (a.rows + 15) / 16 * blocks;
  if (n >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;  // (rows of more than a card holds)
  constexpr int64_t kMost = 1 << 23;  // workgroups of a launch
  for (int64_t first = 0; first < n; first += kMost) {
    const dim3 grid((uint32_t)std::min(n - first, kMost));
    const uint32_t f = (uint32_t)first, nb = (uint32_t)blocks, nt = (uint32_t)tiles;
    if (tile && prec == PACK_PREC_BF16)
      hipLaunchKernelGGL((tile_codes_kernel<__bf16>), grid, dim3(256), 0, s, a, nb, nt, f);
    else if (tile)
      hipLaunchKernelGGL((tile_codes_kernel<float>), grid, dim3(256), 0, s, a, nb, nt, f);
    else if (prec == PACK_PREC_BF16)
      hipLaunchKernelGGL((row_codes_kernel<__bf16>), grid, dim3(256), 0, s, a, nb, f);
    else
      hipLaunchKernelGGL((row_codes_kernel<float>), grid, dim3(256), 0, s, a, nb, f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace tabpack
