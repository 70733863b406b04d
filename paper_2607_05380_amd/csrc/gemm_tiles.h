// Tile primitives shared by the matrix-product kernels (kernels_gemm.hip,
// kernels_block.hip): waits, buffer descriptors, direct-to-LDS loads, the two
// LDS layouts of bf16 operand tiles and their fragment reads.
#pragma once
#include "pack_internal.h"

namespace tabpack {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// depth-contiguous bf16 layout used with direct-to-LDS loads, for K steps of
// KS 16-deep MFMA steps: row-major, 32*KS bytes (CPR = 2*KS 16-byte chunks) of
// depth per row, chunk c of row r stored at chunk position c ^ f(r) with
// f(r) = (r / (16/CPR)) % CPR.  The 16 rows read by a quarter-wave's 16-byte
// fragment loads then cover all 64 banks, and each quad of lanes of a direct
// load fills one aligned 64-byte piece of one row, i.e. it reads one aligned
// 64-byte piece of one global row (in permuted order): one cache-line lookup
// per quad.
template <int KS>
__device__ __forceinline__ int kmaj_f(int row) {
  constexpr int CPR = 2 * KS;
  return (row / (16 / CPR)) & (CPR - 1);
}
template <int KS>
__device__ __forceinline__ int kmaj16_off(int row, int c) {
  return row * (32 * KS) + ((c ^ kmaj_f<KS>(row)) << 4);
}

// rows-contiguous bf16 layout (R rows): the 32-byte chunk c of depth row k at
// chunk position c ^ rmaj_x(k).  The four depth rows a transposing read covers
// then fall on disjoint banks: rows of 256 bytes or more share their banks and
// take four positions, the 128-byte rows of 64-row tiles alternate between the
// two halves of the banks and take two.
template <int R>
__device__ __forceinline__ int rmaj_x(int k) {
  return R >= 128 ? (k & 3) << 1 : ((k >> 1) & 1) << 1;
}
// byte offset of element `col` of depth row k
template <int R>
__device__ __forceinline__ int rmaj_off(int k, int col) {
  return k * (R * 2) + (((col >> 4) ^ rmaj_x<R>(k)) << 5) + ((col & 15) << 1);
}

// ------------------------------------------------------------------ waits --
// vmcnt <= N, every other counter at its maximum (gfx9 s_waitcnt encoding),
// plus lgkmcnt(0) when LDS is set.
template <int N, bool LDS>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((LDS ? 0 : 15) << 8) | ((N >> 4) << 14));
}

// Workgroup barrier without a memory fence: the waits that make data visible
// are explicit around it, and the empty asm statements keep the compiler from
// moving memory accesses across it.
__device__ __forceinline__ void bar() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Global-memory views of pointers taken from the descriptor tables.  The
// compiler cannot infer their address space and would use flat accesses,
// which also count against the LDS counter: every LDS wait of the epilogue
// would then wait for the global stores before it too.
#define TABPACK_GLOBAL __attribute__((address_space(1)))
template <typename V>
__device__ __forceinline__ TABPACK_GLOBAL V* glob(V* p) {
  return (TABPACK_GLOBAL V*)p;
}
template <typename V>
__device__ __forceinline__ const TABPACK_GLOBAL V* glob(const V* p) {
  return (const TABPACK_GLOBAL V*)p;
}

// ------------------------------------------------------- buffer addressing --
constexpr uint32_t kOob = 0x80000000u;   // an offset outside every operand buffer
static_assert(kOperandBytes + 16 == (int64_t)kOob, "operands end below the offset that stands for outside");
constexpr int kRsrcWord3 = 0x00020000;   // gfx9 raw buffer descriptor: 32-bit data format, no swizzle

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(bytes < kOob ? bytes : kOob - 16),
                                           kRsrcWord3);
}

__device__ __forceinline__ u32x4 buf_load16(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
}

typedef void __attribute__((address_space(3)))* lptr_t;
typedef __attribute__((address_space(3))) int32_t lds_i32;

__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, char* lds, uint32_t voff, uint32_t soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)lds, 16, voff, soff, 0, 0);
}

// ------------------------------------------------------------- fragments --
// 8 bf16 of depth 16*ks + 8*h .. +7 (h = lane / 32) of operand row
// row_block + lane % 32, from the rows-contiguous (frag_tr_asm) and the
// depth-contiguous layout, through inline assembly.  The compiler cannot prove
// that a read of one stage does not alias the direct-to-LDS loads just
// issued into the other, and would wait for those loads before every read;
// through assembly the read is invisible to it, so the caller waits for the
// result itself (an explicit lgkmcnt before the first use).
template <int R>
__device__ __forceinline__ u32x2 ds_tr16_b64(const char* p) {
  typedef __attribute__((address_space(3))) const char* lds_cptr;
  const uint32_t a = (uint32_t)(uintptr_t)(lds_cptr)p;
  u32x2 r;
  asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(r) : "v"(a));
  return r;
}
template <int R>
__device__ __forceinline__ bf16x8 frag_tr_asm(const char* lds, int row_block, int ks, int lane) {
  const int s = lane & 15, g = lane >> 4;
  const int k = 16 * ks + 8 * (g >> 1) + (s >> 2);
  const int col = row_block + 16 * (g & 1) + 4 * (s & 3);
  const u32x2 a = ds_tr16_b64<R>(lds + rmaj_off<R>(k, col));
  const u32x2 b = ds_tr16_b64<R>(lds + rmaj_off<R>(k + 4, col));
  return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}

template <int KS>
__device__ __forceinline__ bf16x8 frag_kmaj_asm(const char* lds, int row_block, int ks, int lane) {
  typedef __attribute__((address_space(3))) const char* lds_cptr;
  const uint32_t a = (uint32_t)(uintptr_t)(lds_cptr)(lds + kmaj16_off<KS>(row_block + (lane & 31), 2 * ks + (lane >> 5)));
  u32x4 r;
  asm volatile("ds_read_b128 %0, %1" : "=v"(r) : "v"(a));
  return __builtin_bit_cast(bf16x8, r);
}

}  // namespace
}  // namespace tabpack
