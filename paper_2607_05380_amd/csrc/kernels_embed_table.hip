// Lookup in a table of embeddings and the table's gradient, on gfx950.
//
// Forward: y[t] = scale table[idx[t]].  A thread takes one vector of 16 bytes;
// bandwidth bounds it.
//
// Backward: dtable[v] = scale sum over the t with idx[t] = v of dy[t].  The
// tokens are sorted by index, stably, so that each row's tokens lie together in
// the order of the batch; chunks of the sorted list are then summed in fp32 by
// groups of threads that own columns, dy's rows read once each.  A row of
// few tokens is written from its registers; parts of one that takes several chunks go
// to memory and a last kernel adds them up in a fixed order.  No atomics
// on sums, so the result does not change between runs.  Rows that no token names
// are zeros, written while the sort runs (it occupies a few CUs and is
// latency; the table's bytes are bandwidth).
//
// The sort is by digits of the index from the lowest on.  A wave ranks 64 tokens
// at a time: lanes with the same digit find each other by ballots, one of them
// advances the wave's count of the digit.  Up to 4096 tokens one workgroup holds
// all of them in registers and LDS, and one launch sorts (16,384 that way took
// 34 us, in 64 workgroups 24); longer lists take two launches a digit or three.
//
// Measured: 65,536 tokens of 100,003 x 512 bf16 looked up in 18 us; the gradient
// of 16,384 tokens of 32,000 x 1024 bf16 47 us (sort and zeros 24, six launches of 5
// to 8 us; sums 15, at 3.3 TB/s; join 8), of 1,000,000 tokens of 1600 x 32 fp32 72 (count 8, scan 4,
// move 16, sums 32, at 4.1 TB/s of gathered rows of 128 bytes, join 11).
#include <algorithm>

#include "ops_internal.h"
#include "row_tiles.h"
#include "../../include/tabpack.h"

namespace tabpack {
namespace {

// The row that token t names: -1 none, `rows` one that is not there.
__device__ __forceinline__ int64_t row_of(const void* idx, int idx64, int64_t t, int64_t rows) {
  const int64_t i = idx64 ? static_cast<const int64_t*>(idx)[t] : static_cast<const int32_t*>(idx)[t];
  return i < 0 ? -1 : i < rows ? i : rows;
}

// ---------------------------------------------------------------- forward --
template <typename T, typename I>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, I vectors, I total) {
  constexpr int VE = kVec<T>;
  for (I i = (I)blockIdx.x * 256 + threadIdx.x; i < total; i += (I)gridDim.x * 256) {
    const I t = i / vectors;
    const int c = (int)(i - t * vectors) * VE, n = a.cols - c;
    const int64_t row = row_of(a.idx, a.idx64, (int64_t)t, a.rows);
    float v[VE];
    if (row >= 0 && row < a.rows) {
      Vec<T> x;
      x.load(static_cast<const T*>(a.table) + row * a.ldt + c, n);
      x.get(v);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] *= a.scale;
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = row < 0 ? 0.0f : __builtin_nanf("");
    }
    store_vec(static_cast<T*>(a.out) + (int64_t)t * a.ldo + c, v, n);
  }
}

template <typename T>
hipError_t embed_t(const EmbedArgs& a, hipStream_t s) {
  const int64_t vectors = ((int64_t)a.cols + kVec<T> - 1) / kVec<T>, total = a.tokens * vectors;
  const dim3 grid(row_blocks(total, 256));
  // (32-bit divisions where they do)
  if (total < (int64_t)1 << 31)
    hipLaunchKernelGGL((embed_kernel<T, uint32_t>), grid, dim3(256), 0, s, a, (uint32_t)vectors, (uint32_t)total);
  else
    hipLaunchKernelGGL((embed_kernel<T, uint64_t>), grid, dim3(256), 0, s, a, (uint64_t)vectors, (uint64_t)total);
  return hipGetLastError();
}

// ------------------------------------------------------------------- sort --
constexpr uint32_t kNoKey = 0xffffffffu;  // places behind the last token: after every key

// A token of the list: its key, and its place in the batch (one store moves both).
struct alignas(8) Token {
  uint32_t key, place;
};

// The tokens first + stride j of the batch (past its end: some token's key).  A
// key is the row, or `rows` for a token that adds to none.
template <int N>
__device__ __forceinline__ void keys_of(const EmbedBwdArgs& a, int64_t first, int stride, Token (&t)[N]) {
  int64_t row[N];
  if (a.idx64) {
#pragma unroll
    for (int j = 0; j < N; ++j) row[j] = static_cast<const int64_t*>(a.idx)[min(first + stride * j, a.tokens - 1)];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) row[j] = static_cast<const int32_t*>(a.idx)[min(first + stride * j, a.tokens - 1)];
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    t[j] = Token{(uint32_t)(row[j] < 0 || row[j] >= a.rows ? a.rows : row[j]), (uint32_t)(first + stride * j)};
}

__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The wave's next 64 keys' digits d: how many of the wave's keys before this one
// have it.  count: the wave's counts, 1 << DB.
template <int DB, typename C>
__device__ __forceinline__ uint32_t rank_digit(uint32_t d, C* count, int lane) {
  uint64_t same = ~0ull;
#pragma unroll
  for (int b = 0; b < DB; ++b) {
    const bool one = (d >> b) & 1;
    const uint64_t ones = __ballot(one);
    same &= one ? ones : ~ones;
  }
  const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1));
  const uint32_t base = count[d];
  wave_order();
  if (before == 0) count[d] = (C)(base + (uint32_t)__popcll(same));
  wave_order();
  return base + before;
}

// Exclusive running sum over the block's first N threads (N / 64 whole waves);
// waves: LDS of N / 64 words.  Every thread of the block calls it.
template <int N>
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t v, uint32_t* waves, int tid) {
  uint32_t s = v;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t o = __shfl_up(s, m, 64);
    if ((tid & 63) >= m) s += o;
  }
  if (tid < N && (tid & 63) == 63) waves[tid >> 6] = s;
  __syncthreads();
  uint32_t before = s - v;
  if (tid < N)
    for (int w = 0; w < tid >> 6; ++w) before += waves[w];
  __syncthreads();
  return before;
}

// Zeros over part `part` of `parts` of the table, by block `block` of `blocks` of NT threads.
template <typename T, int NT>
__device__ __forceinline__ void fill(const EmbedBwdArgs& a, uint32_t block, uint32_t blocks, int part = 0,
                                     int parts = 1) {
  constexpr int VE = kVec<T>;
  const int64_t each = (a.rows * a.cols / parts / VE + 1) * VE, n = min(a.rows * a.cols, (part + 1) * each);
  T* const p = static_cast<T*>(a.dtable);
  float zero[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) zero[e] = 0.0f;
  for (int64_t i = part * each + ((int64_t)block * NT + threadIdx.x) * VE; i < n; i += (int64_t)blocks * NT * VE)
    store_vec(p + i, zero, (int)(n - i < VE ? n - i : VE));
}

// Up to 1024 IPT tokens in one workgroup (block 0; the others write zeros).
template <typename T, int IPT>
__global__ __launch_bounds__(1024) void sort_one_kernel(EmbedBwdArgs a, Token* list, int bits) {
  __shared__ uint32_t lds_key[1024 * IPT], lds_place[1024 * IPT], count[16][256], waves[4];
  if (blockIdx.x > 0) {
    fill<T, 1024>(a, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = (int)a.tokens;
  const int first = wave * 64 * IPT + lane;  // the thread's items: first + 64 j
  uint32_t key[IPT], place[IPT], rank[IPT];
  if (n > 0) {
    Token t[IPT];
    keys_of<IPT>(a, first, 64, t);
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      key[j] = first + 64 * j < n ? t[j].key : kNoKey;
      place[j] = t[j].place;
    }
  } else {
#pragma unroll
    for (int j = 0; j < IPT; ++j) key[j] = kNoKey, place[j] = 0;
  }
  for (int shift = 0; shift < bits; shift += 8) {
    for (int i = tid; i < 16 * 256; i += 1024) count[i >> 8][i & 255] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < IPT; ++j) rank[j] = rank_digit<8>((key[j] >> shift) & 255, count[wave], lane);
    __syncthreads();
    // the place of each wave's first key of a digit: behind all lower digits and the waves before
    uint32_t total = 0;
    if (tid < 256)
      for (int w = 0; w < 16; ++w) {
        const uint32_t c = count[w][tid];
        count[w][tid] = total;
        total += c;
      }
    const uint32_t before = exclusive_sum<256>(total, waves, tid);
    if (tid < 256)
      for (int w = 0; w < 16; ++w) count[w][tid] += before;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      const uint32_t to = count[wave][(key[j] >> shift) & 255] + rank[j];
      lds_key[to] = key[j];
      lds_place[to] = place[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      key[j] = lds_key[first + 64 * j];
      place[j] = lds_place[first + 64 * j];
    }
    // (the next round's counts are cleared behind these reads' barriers)
  }
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int i = first + 64 * j;
    if (i < n) list[i] = Token{key[j], place[j]};
  }
}

// Longer lists, a digit of DB bits in two launches or three: blocks of NT IPT
// tokens count theirs, then move them.  Up to kDirect blocks of 256 threads (65,536
// tokens) a move adds up the counts of the blocks before its own by itself; blocks
// of 1024 threads take a launch between for that (65,536 tokens of 200,000 x 128 in
// 16 of them 61 us, in 64 small ones 45; each block counting the whole list instead
// of a launch for the counts: 16,384 tokens of 32,000 x 1024 49 us, this way 47).  The
// blocks behind the sort's write zeros.  What bounds the moves of a long list is its
// scattered stores: larger blocks have longer runs of a digit.
constexpr uint32_t kDirect = 64;
struct SortArgs {
  const Token* list;
  Token* out;
  uint32_t* counts;  // small blocks: [blocks, digits]; large ones: [digits, blocks], behind a scan those before
  uint32_t* totals;  // [digits] (with a scan)
  uint32_t blocks;
  int shift, round, launch, launches;  // (launches: those that write zeros)
};
// The tokens first + stride j, all of them asked for together (past the end:
// kNoKey).  The lists hold one token at least.
template <int N>
__device__ __forceinline__ void sort_tokens(const EmbedBwdArgs& a, const SortArgs& s, int64_t first, int stride,
                                            Token (&t)[N]) {
  if (s.round) {
#pragma unroll
    for (int j = 0; j < N; ++j) t[j] = s.list[min(first + stride * j, a.tokens - 1)];
  } else {
    keys_of<N>(a, first, stride, t);
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (first + stride * j >= a.tokens) t[j].key = kNoKey;
}
template <typename T, int DB, int NT, int IPT>
__global__ __launch_bounds__(NT) void sort_count_kernel(EmbedBwdArgs a, SortArgs s) {
  __shared__ uint32_t count[1 << DB];
  if (blockIdx.x >= s.blocks) {
    fill<T, NT>(a, blockIdx.x - s.blocks, gridDim.x - s.blocks, s.launch, s.launches);
    return;
  }
  for (int d = threadIdx.x; d < 1 << DB; d += NT) count[d] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * (NT * IPT) + threadIdx.x;
  Token token[IPT];
  sort_tokens(a, s, first, NT, token);
#pragma unroll
  for (int j = 0; j < IPT; ++j)  // (whole numbers: the order of these additions does not matter)
    if (token[j].key != kNoKey) atomicAdd(&count[(token[j].key >> s.shift) & ((1 << DB) - 1)], 1u);
  __syncthreads();
  // (in the order in which a move, or the scan, reads them)
  const int64_t of_digit = NT == 256 ? 1 : s.blocks, of_block = NT == 256 ? 1 << DB : 1;
  for (int d = threadIdx.x; d < 1 << DB; d += NT) s.counts[d * of_digit + blockIdx.x * of_block] = count[d];
}
// A block: one digit's counts over the blocks of tokens, to those of the blocks before each.
__global__ __launch_bounds__(256) void sort_scan_kernel(SortArgs s) {
  __shared__ uint32_t waves[4], last;
  uint32_t* const c = s.counts + (int64_t)blockIdx.x * s.blocks;
  uint32_t carry = 0;
  for (uint32_t base = 0; base < s.blocks; base += 256) {
    const uint32_t i = base + threadIdx.x, v = i < s.blocks ? c[i] : 0;
    const uint32_t before = exclusive_sum<256>(v, waves, threadIdx.x);
    if (i < s.blocks) c[i] = carry + before;
    if (threadIdx.x == 255) last = before + v;
    __syncthreads();
    carry += last;
    __syncthreads();
  }
  if (threadIdx.x == 0) s.totals[blockIdx.x] = carry;
}
template <typename T, int DB, int NT, int IPT, bool DIRECT>
__global__ __launch_bounds__(NT) void sort_move_kernel(EmbedBwdArgs a, SortArgs s) {
  constexpr int D = 1 << DB, W = NT / 64, PER = D / NT > 0 ? D / NT : 1;
  __shared__ __attribute__((aligned(16))) uint16_t count[W][D];  // of each wave, at most 64 IPT
  __shared__ uint32_t base[D], waves[W];
  if (blockIdx.x >= s.blocks) {
    fill<T, NT>(a, blockIdx.x - s.blocks, gridDim.x - s.blocks, s.launch, s.launches);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < W * D / 2; i += NT) reinterpret_cast<uint32_t*>(&count[0][0])[i] = 0;
  const int64_t first = (int64_t)blockIdx.x * (NT * IPT) + wave * (64 * IPT) + lane;
  Token token[IPT];
  uint32_t rank[IPT];
  sort_tokens(a, s, first, 64, token);
  // a thread's PER digits: tokens with the digit, and those of the blocks before
  uint32_t total[PER], before[PER], sum = 0;
  const bool has = tid * PER < D;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    total[q] = before[q] = 0;
    const int d = has ? tid * PER + q : 0;
    if constexpr (DIRECT) {
      for (uint32_t b0 = 0; b0 < s.blocks; b0 += 32) {
        uint32_t n[32];
#pragma unroll
        for (uint32_t u = 0; u < 32; ++u) n[u] = s.counts[min(b0 + u, s.blocks - 1) * D + d];
#pragma unroll
        for (uint32_t u = 0; u < 32; ++u) {
          total[q] += b0 + u < s.blocks ? n[u] : 0;
          before[q] += b0 + u < blockIdx.x ? n[u] : 0;
        }
      }
    } else {
      total[q] = s.totals[d];
      before[q] = s.counts[(int64_t)d * s.blocks + blockIdx.x];
    }
    if (!has) total[q] = 0;
    sum += total[q];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < IPT; ++j) rank[j] = rank_digit<DB>((token[j].key >> s.shift) & (D - 1), count[wave], lane);
  // where the block's first token of a digit goes, behind the lower digits and the blocks before; each wave's
  // behind those of the waves before
  uint32_t lower = exclusive_sum<NT>(sum, waves, tid);  // (its barriers stand behind the ranks)
  if (has) {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      base[tid * PER + q] = lower + before[q];
      lower += total[q];
      uint32_t at = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const uint32_t c = count[w][tid * PER + q];
        count[w][tid * PER + q] = (uint16_t)at;
        at += c;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    if (first + 64 * j >= a.tokens) continue;
    const uint32_t d = (token[j].key >> s.shift) & (D - 1);
    s.out[base[d] + count[wave][d] + rank[j]] = token[j];
  }
}

// ------------------------------------------------------------------- sums --
// A row whose tokens begin in a chunk and end in it or in the next one is its
// chunk's alone: the group that has its beginning goes on into the next chunk, whose
// group leaves them out.  Longer rows have a part of each chunk: the one where they
// begin, and those that they pass through or end in.
struct SumArgs {
  const Token* list;
  // [chunks, 2, ldp]: the part of a chunk's first row, begun before it, and of its last one, which goes on
  float* partial;
  int64_t ldp;
  int32_t chunk;   // tokens of a chunk
  int32_t chunks, g, columns;  // 1 << g threads own a vector of columns each; groups side by side over the columns
  int32_t per;     // chunks that a block of the join looks through
  bool many;       // its blocks have 1024 threads, not 256
};
__device__ __forceinline__ uint32_t key_at(const EmbedBwdArgs& a, const SumArgs& s, int64_t i) {
  return i < 0 || i >= a.tokens ? kNoKey : s.list[i].key;  // (kNoKey: no token's)
}
// Whether the row of the chunk's last token goes on behind it, and as a long one,
// and whether it begins in the chunk.
struct Tail {
  uint32_t key;
  bool open, starts, lasts;  // into the next chunk; in this one; past the next one
  __device__ __forceinline__ Tail(const EmbedBwdArgs& a, const SumArgs& s, int64_t chunk) {
    const int64_t i0 = chunk * s.chunk, i1 = i0 + s.chunk;
    const uint32_t before = key_at(a, s, i0 - 1), after = key_at(a, s, i1), past = key_at(a, s, i1 + s.chunk);
    key = key_at(a, s, i1 - 1);
    open = key < a.rows && after == key;
    starts = before != key;  // (sorted: if the token before the chunk has it, the whole chunk has)
    lasts = past == key;
  }
};

template <typename T>
__device__ __forceinline__ void write_row(const EmbedBwdArgs& a, uint32_t key, int c, const float* acc) {
  float v[kVec<T>];
#pragma unroll
  for (int e = 0; e < kVec<T>; ++e) v[e] = acc[e] * a.scale;
  store_vec(static_cast<T*>(a.dtable) + (int64_t)key * a.cols + c, v, a.cols - c);
}

template <typename T>
__global__ __launch_bounds__(256) void run_sum_kernel(EmbedBwdArgs a, SumArgs s) {
  constexpr int VE = kVec<T>, U = 8;
  const int64_t unit = (int64_t)blockIdx.x * (256 >> s.g) + (threadIdx.x >> s.g);
  const int64_t chunk = unit / s.columns;
  if (chunk >= s.chunks) return;
  const int c = (((int)(unit % s.columns) << s.g) + (threadIdx.x & ((1 << s.g) - 1))) * VE;
  const int n = a.cols - c;
  if (n <= 0) return;
  const int64_t i0 = chunk * s.chunk, i1 = min(a.tokens, i0 + s.chunk);
  Token token[U];  // the next U
  auto ask = [&](int64_t i) {
#pragma unroll
    for (int u = 0; u < U; ++u) token[u] = s.list[min(i + u, a.tokens - 1)];
  };
  ask(i0);
  const Tail tail(a, s, chunk);
  // the first tokens' row begun before: the chunk before's own, or one with a part here
  const uint32_t first = token[0].key, before = key_at(a, s, i0 - 1);
  const bool begun = before == first;
  const bool skip = begun && (tail.key != first || !tail.open) && key_at(a, s, i0 - s.chunk - 1) != first;
  // a short row at the end is followed into the next chunk
  const bool follow = tail.open && tail.starts && !tail.lasts;
  const int64_t end = follow ? min(a.tokens, i1 + s.chunk) : i1;
  float* const partial = s.partial + chunk * 2 * s.ldp + c;
  const T* const dy = static_cast<const T*>(a.dy) + c;
  uint32_t cur = first;
  bool head = begun;  // the present row was begun before the chunk
  float acc[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
  auto flush = [&] {  // the present row has ended
    if (!head) {
      write_row<T>(a, cur, c, acc);
    } else if (!skip) {
#pragma unroll
      for (int e = 0; e < VE; ++e) partial[e] = acc[e];
    }
  };
  for (int64_t i = i0; i < end; i += U) {
    uint32_t key[U];
    Vec<T> v[U];
    // (every place is a token's: what is read of rows that are not this group's to add is not used)
    if (n >= VE) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u].raw = *reinterpret_cast<const u32x4_any*>(dy + (int64_t)token[u].place * a.ldy);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u].load(dy + (int64_t)token[u].place * a.ldy, n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) key[u] = token[u].key;
    if (i + U < end) ask(i + U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= end) break;
      if (key[u] != cur) {
        flush();
        if (i + u >= i1 || key[u] >= a.rows) return;  // (the followed row's end; those without a row come last)
        cur = key[u];
        head = false;
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
      }
      if (cur >= a.rows) return;
      float x[VE];
      v[u].get(x);
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[e] += x[e];
    }
  }
  if (follow || !tail.open) {
    flush();
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) partial[(head ? 0 : s.ldp) + e] = acc[e];
  }
}

// A block: the long rows that begin in its chunks, for one group of columns, one
// after the other.  Its threads' groups take a row's chunks in turn.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void run_join_kernel(EmbedBwdArgs a, SumArgs s) {
  constexpr int VE = kVec<T>, B = NT > 256 ? 32 / VE : 4;
  __shared__ float part[NT][VE + 1];
  __shared__ uint32_t key_of_chunk[16];
  const int64_t first = (int64_t)(blockIdx.x / s.columns) * s.per;
  if (threadIdx.x < (uint32_t)s.per) {
    const Tail t(a, s, first + threadIdx.x);
    key_of_chunk[threadIdx.x] = t.open && t.starts && t.lasts ? t.key : kNoKey;
  }
  __syncthreads();
  const int lane = threadIdx.x & ((1 << s.g) - 1), group = threadIdx.x >> s.g, groups = NT >> s.g;
  const int c = (((int)(blockIdx.x % s.columns) << s.g) + lane) * VE;
  for (int q = 0; q < s.per; ++q) {
    const uint32_t key = key_of_chunk[q];
    if (key == kNoKey) continue;  // (the same for the whole block)
    const int64_t chunk = first + q;
    float acc[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
    if (c < a.cols) {
      if (group == 0) {
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] = s.partial[(chunk * 2 + 1) * s.ldp + c + e];
      }
      // the next B chunks' first keys and sums are asked for together
      bool more = true;
      for (int64_t b0 = chunk + 1 + group; more; b0 += (int64_t)B * groups) {
        bool goes[B];
        f32x4 v[B][VE / 4];
#pragma unroll
        for (int u = 0; u < B; ++u) {
          const int64_t b = min(b0 + (int64_t)u * groups, (int64_t)s.chunks - 1);
          goes[u] = b0 + (int64_t)u * groups < s.chunks && s.list[b * s.chunk].key == key;
#pragma unroll
          for (int h = 0; h < VE / 4; ++h)
            v[u][h] = *reinterpret_cast<const f32x4*>(s.partial + b * 2 * s.ldp + c + 4 * h);
        }
#pragma unroll
        for (int u = 0; u < B; ++u) {
#pragma unroll
          for (int e = 0; e < VE; ++e) acc[e] += goes[u] ? v[u][e / 4][e % 4] : 0.0f;
        }
        more = goes[B - 1];
      }
    }
    // the groups' sums by halves
    for (int h = groups / 2; h >= 1; h /= 2) {
#pragma unroll
      for (int e = 0; e < VE; ++e) part[threadIdx.x][e] = acc[e];
      __syncthreads();
      if (group < h) {
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] += part[((group + h) << s.g) + lane][e];
      }
      __syncthreads();
    }
    if (group == 0 && c < a.cols) write_row<T>(a, key, c, acc);
  }
}

// ------------------------------------------------------------------- host --
constexpr int64_t kSortOne = 4096;  // tokens that one workgroup sorts

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// How a gradient is laid out over launches, and its workspace.
struct BwdPlan {
  int bits, digit, rounds;  // of the keys, of a digit, digits
  int tile;                 // tokens of a block of the long sort
  uint32_t blocks;          // of tokens in the long sort
  SumArgs sum;
  size_t counts, totals, partial, bytes;  // byte offsets
};
BwdPlan plan(int prec, int64_t tokens, int64_t rows, int32_t cols) {
  BwdPlan p{};
  const int ve = prec == PACK_PREC_BF16 ? 8 : 4;
  while (p.bits < 32 && (rows >> p.bits) > 0) ++p.bits;  // keys 0 .. rows
  const bool one = tokens <= kSortOne;
  p.tile = tokens <= 256 * (int64_t)kDirect ? 256 : tokens <= 1024 * (int64_t)kDirect ? 1024 : 4096;
  p.blocks = one ? 0 : (uint32_t)((tokens + p.tile - 1) / p.tile);
  // digits of 8 bits, or in the largest blocks of 11 where that saves a round
  p.digit = p.tile == 4096 && (p.bits + 10) / 11 < (p.bits + 7) / 8 ? 11 : 8;
  p.rounds = (p.bits + p.digit - 1) / p.digit;
  const int64_t vectors = ((int64_t)cols + ve - 1) / ve;
  while (p.sum.g < 6 && ((int64_t)1 << p.sum.g) < vectors) ++p.sum.g;
  p.sum.columns = (int)((vectors + (1 << p.sum.g) - 1) >> p.sum.g);
  // chunks for some 4096 waves (1,000,000 tokens of 1600 x 32 fp32: as fast with 2048, 8192 3 us slower), of 16 to
  // 1024 tokens; larger ones where rows have thousands of chunks, whose parts are joined one after the other
  int64_t chunk = 16;
  while (chunk < 1024 && tokens * p.sum.columns * (1 << p.sum.g) / 64 > 4096 * chunk) chunk *= 2;
  while (chunk < 128 && tokens > 4096 * chunk * rows) chunk *= 2;
  p.sum.chunk = (int)chunk;
  p.sum.chunks = (int)((tokens + chunk - 1) / chunk);
  p.sum.ldp = vectors * ve;
  // blocks of the join: as many as the chip holds at a time, of 1 to 16 chunks; large ones where a row takes
  // many threads, or has hundreds of chunks (1,000,000 tokens of 2 x 32 fp32 69 us; in chunks of 32 103, and with
  // 256 threads 255)
  p.sum.many = p.sum.g >= 5 || tokens > 256 * chunk * rows;
  p.sum.per = 1;
  const int64_t held = p.sum.many ? 512 : 4096;
  while (p.sum.per < 16 && (int64_t)p.sum.chunks * p.sum.columns > held * p.sum.per) p.sum.per *= 2;
  size_t at = (size_t)up(tokens * 8, 16) * (one ? 1 : 2);
  p.counts = at;
  at += (size_t)up(((int64_t)p.blocks << p.digit) * 4, 16);
  p.totals = at;
  at += one || p.tile < 4096 ? 0 : (size_t)4 << p.digit;
  p.partial = at;
  if (p.sum.chunks > 1) at += (size_t)p.sum.chunks * 2 * (size_t)p.sum.ldp * 4;
  p.bytes = at;
  return p;
}

// The list ends up in buf[(rounds + 1) & 1].
template <typename T, int DB, int NT, int IPT>
hipError_t sort_long(const EmbedBwdArgs& a, const BwdPlan& p, SortArgs s, Token* const (&buf)[2], hipStream_t st) {
  s.launches = 2 * p.rounds;
  // blocks that write zeros: a KB a wave and launch or more, up to four blocks a CU
  const int64_t bytes = a.rows * a.cols * (int64_t)sizeof(T) / s.launches, each = NT * 16;
  const dim3 grid(p.blocks + (uint32_t)std::min<int64_t>((bytes + each - 1) / each, 1024)), block(NT);
  for (s.round = 0; s.round < p.rounds; ++s.round) {
    s.shift = s.round * DB;
    s.list = buf[(s.round + 1) & 1], s.out = buf[s.round & 1];
    s.launch = 2 * s.round;
    hipLaunchKernelGGL((sort_count_kernel<T, DB, NT, IPT>), grid, block, 0, st, a, s);
    ++s.launch;
    if constexpr (NT == 256) {  // (up to kDirect blocks)
      hipLaunchKernelGGL((sort_move_kernel<T, DB, NT, IPT, true>), grid, block, 0, st, a, s);
    } else {
      hipLaunchKernelGGL(sort_scan_kernel, dim3(1 << DB), dim3(256), 0, st, s);
      hipLaunchKernelGGL((sort_move_kernel<T, DB, NT, IPT, false>), grid, block, 0, st, a, s);
    }
  }
  return hipGetLastError();
}

template <typename T>
hipError_t embed_bwd_t(int prec, const EmbedBwdArgs& a, hipStream_t st) {
  const BwdPlan p = plan(prec, a.tokens, a.rows, a.cols);
  if ((int64_t)p.sum.chunks * p.sum.columns >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;  // (2^32 threads)
  char* const w = static_cast<char*>(a.work);
  Token* const buf[2] = {reinterpret_cast<Token*>(w), reinterpret_cast<Token*>(w + up(a.tokens * 8, 16))};
  hipError_t e;
  int last = 0;  // the buffer that holds the sorted list
  if (a.tokens <= kSortOne) {
    const int64_t bytes = a.rows * a.cols * (int64_t)sizeof(T);
    const dim3 grid(1 + (uint32_t)std::min<int64_t>((bytes + 65535) / 65536, 512)), block(1024);
    if (a.tokens <= 1024)
      hipLaunchKernelGGL((sort_one_kernel<T, 1>), grid, block, 0, st, a, buf[0], p.bits);
    else
      hipLaunchKernelGGL((sort_one_kernel<T, 4>), grid, block, 0, st, a, buf[0], p.bits);
    e = hipGetLastError();
  } else {
    SortArgs s{};
    s.counts = reinterpret_cast<uint32_t*>(w + p.counts), s.totals = reinterpret_cast<uint32_t*>(w + p.totals);
    s.blocks = p.blocks;
    if (p.tile == 256)
      e = sort_long<T, 8, 256, 1>(a, p, s, buf, st);
    else if (p.tile == 1024)
      e = sort_long<T, 8, 256, 4>(a, p, s, buf, st);
    else
      e = p.digit == 8 ? sort_long<T, 8, 1024, 4>(a, p, s, buf, st) : sort_long<T, 11, 1024, 4>(a, p, s, buf, st);
    last = (p.rounds + 1) & 1;
  }
  if (e != hipSuccess || a.tokens == 0) return e;
  SumArgs s = p.sum;
  s.list = buf[last];
  s.partial = reinterpret_cast<float*>(w + p.partial);
  const int64_t units = (int64_t)s.chunks * s.columns, per = 256 >> s.g;
  hipLaunchKernelGGL((run_sum_kernel<T>), dim3((uint32_t)((units + per - 1) / per)), dim3(256), 0, st, a, s);
  if (s.chunks > 2) {  // (a row over two chunks is short)
    const int64_t joins = ((int64_t)s.chunks + s.per - 1) / s.per * s.columns;
    if (s.many)
      hipLaunchKernelGGL((run_join_kernel<T, 1024>), dim3((uint32_t)joins), dim3(1024), 0, st, a, s);
    else
      hipLaunchKernelGGL((run_join_kernel<T, 256>), dim3((uint32_t)joins), dim3(256), 0, st, a, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(int prec, const EmbedArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? embed_t<__bf16>(a, s) : embed_t<float>(a, s);
}

size_t embed_bwd_bytes(int prec, int64_t tokens, int64_t rows, int32_t cols) {
  return plan(prec, tokens, rows, cols).bytes;
}

hipError_t launch_embed_bwd(int prec, const EmbedBwdArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? embed_bwd_t<__bf16>(prec, a, s) : embed_bwd_t<float>(prec, a, s);
}

}  // namespace tabpack
