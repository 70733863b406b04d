// Dropout whose mask is never stored, on gfx950: y = (residual +) x s where the
// element is kept, s = 1 / (1 - p), and residual (or 0) where it is not.  The
// backward pass is the same call on dy.
//
// Element (r, c) takes the 16-bit half c % 2 of word (c / 2) % 4 of the Philox
// block with counter (c / 8, r, site, step) and is kept if the half is at least
// floor(p 2^16) (so the share kept is 1 - p rounded up to a multiple of 2^-16): the
// packs' rule, one block for 8 neighbours of a row, which are
// one or two vectors of a thread.  The draws depend on (r, c) alone, not on how
// the tensor lies or how threads share it.  A block costs some 90 instructions for
// 8 elements, close to what their bytes take in HBM, which bounds it: 65,536 x
// 1024 bf16 71 us with a residual (5.7 TB/s), 47 without (5.7).
#include "ops_internal.h"
#include "philox.h"
#include "row_tiles.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

template <typename T, typename I>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, I groups, I total) {
  constexpr int VE = kVec<T>, NV = 8 / VE;
  const uint32_t step = a.step_at ? (uint32_t)*a.step_at : a.step;
  for (I i = (I)blockIdx.x * 256 + threadIdx.x; i < total; i += (I)gridDim.x * 256) {
    const I row = i / groups;
    const uint32_t group = (uint32_t)(i - row * groups);
    const int c = (int)group * 8, n = a.cols - c;
    Vec<T> xs[NV], rs[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      xs[q].load(static_cast<const T*>(a.x) + (int64_t)row * a.ldx + c + q * VE, n - q * VE);
      if (a.residual) rs[q].load(static_cast<const T*>(a.residual) + (int64_t)row * a.ldr + c + q * VE, n - q * VE);
    }
    Words4 w{0, 0, 0, 0};
    if (a.threshold) w = philox4x32_10(group, (uint32_t)row, a.site, step, a.key0, a.key1);
    const uint32_t words[4] = {w.w0, w.w1, w.w2, w.w3};
    T* const out = static_cast<T*>(a.out) + (int64_t)row * a.ldo + c;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      float x[VE], r[VE];
      xs[q].get(x);
      if (a.residual) {
        rs[q].get(r);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) r[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int j = q * VE + e;
        const uint32_t draw = j % 2 ? words[j / 2] >> 16 : words[j / 2] & 0xffffu;
        // (a dropped element is left out whatever it holds)
        x[e] = draw >= a.threshold ? fmaf(x[e], a.scale, r[e]) : r[e];
      }
      store_vec(out + q * VE, x, n - q * VE);
    }
  }
}

template <typename T>
hipError_t dropout_t(const DropoutArgs& a, hipStream_t s) {
  const int64_t groups = ((int64_t)a.cols + 7) / 8, total = a.rows * groups;
  const dim3 grid(row_blocks(total, 256));
  // (32-bit divisions where they do)
  if (total < (int64_t)1 << 31)
    hipLaunchKernelGGL((dropout_kernel<T, uint32_t>), grid, dim3(256), 0, s, a, (uint32_t)groups, (uint32_t)total);
  else
    hipLaunchKernelGGL((dropout_kernel<T, uint64_t>), grid, dim3(256), 0, s, a, (uint64_t)groups, (uint64_t)total);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int prec, const DropoutArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? dropout_t<__bf16>(a, s) : dropout_t<float>(a, s);
}

}  // namespace tabpack
