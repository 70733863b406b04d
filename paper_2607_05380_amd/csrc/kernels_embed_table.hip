// Lookup in a table of embeddings and the table's gradient, on gfx950.
//
// Forward: y[t] = scale table[idx[t]].  A thread takes one vector of 16 bytes;
// bandwidth bounds it.
//
// Backward: dtable[v] = scale sum over the t with idx[t] = v of dy[t].  The
// tokens are sorted by index, stably, so that each row's tokens lie together in
// the order of the batch; chunks of the sorted list are then summed in fp32 by
// groups of threads that own columns, dy's rows read once each.  A row whose
// tokens lie in one chunk is written from its registers; parts of a row that
// crosses chunks go to memory and a last kernel adds them up in order.  No atomics
// on sums, so the result does not change between runs.  Rows that no token names
// are zeros, written while the sort runs (it occupies a few CUs and is
// latency; the table's bytes are bandwidth).
//
// The sort is by digits of the index from the lowest on.  A wave ranks 64 tokens
// at a time: lanes with the same digit find each other by ballots, one of them
// advances the wave's count of the digit.  Up to 16,384 tokens one workgroup holds
// all of them in LDS and one launch sorts; longer lists take three launches a
// digit (counts per block of 4096, their running sums, the move).
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

// A token's key: its row, or `rows` for one that adds to none.
__device__ __forceinline__ uint32_t key_of(const EmbedBwdArgs& a, int64_t t) {
  const int64_t r = row_of(a.idx, a.idx64, t, a.rows);
  return (uint32_t)(r < 0 ? a.rows : r);
}

__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The wave's next 64 keys' digits d: how many of the wave's keys before this one
// have it.  count: the wave's counts, 1 << DB.
template <int DB>
__device__ __forceinline__ uint32_t rank_digit(uint32_t d, uint32_t* count, int lane) {
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
  if (before == 0) count[d] = base + (uint32_t)__popcll(same);
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
__global__ __launch_bounds__(1024) void sort_one_kernel(EmbedBwdArgs a, uint32_t* keys, uint32_t* places, int bits) {
  __shared__ uint32_t lds_key[1024 * IPT], lds_place[1024 * IPT], count[16][256], waves[4];
  if (blockIdx.x > 0) {
    fill<T, 1024>(a, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = (int)a.tokens;
  const int first = wave * 64 * IPT + lane;  // the thread's items: first + 64 j
  uint32_t key[IPT], place[IPT], rank[IPT];
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int i = first + 64 * j;
    key[j] = i < n ? key_of(a, i) : kNoKey;
    place[j] = (uint32_t)i;
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
    if (i < n) keys[i] = key[j], places[i] = place[j];
  }
}

// Longer lists, one digit of DB bits a launch: blocks of 256 IPT tokens.  The
// first launch counts each block's first digits.  A move knows where every token
// goes, so it also counts the next digits of the blocks that it moves them to
// (whole numbers: the order of these additions does not matter).  Up to kDirect
// blocks a move adds up the counts of the blocks before its own by itself, past
// that a launch between them does.  The blocks behind the sort's write zeros.
constexpr uint32_t kDirect = 64;
struct SortArgs {
  const uint32_t* keys;
  const uint32_t* places;
  uint32_t* keys_out;
  uint32_t* places_out;
  uint32_t* counts;        // [digits, blocks] of each block; behind a scan: of the blocks before it
  uint32_t* next;          // the same of the next digit, or NULL
  uint32_t* totals;        // [digits] (with a scan)
  uint32_t blocks;
  int shift, round, rounds;
};
template <typename T, int DB, int IPT>
__global__ __launch_bounds__(256) void sort_count_kernel(EmbedBwdArgs a, SortArgs s) {
  __shared__ uint32_t count[1 << DB];
  if (blockIdx.x >= s.blocks) {
    fill<T, 256>(a, blockIdx.x - s.blocks, gridDim.x - s.blocks, 0, s.rounds + 1);
    return;
  }
  for (int d = threadIdx.x; d < 1 << DB; d += 256) count[d] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * (256 * IPT) + threadIdx.x;
  uint32_t key[IPT];
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int64_t i = first + 256 * j;
    key[j] = i < a.tokens ? key_of(a, i) : kNoKey;
  }
#pragma unroll
  for (int j = 0; j < IPT; ++j)
    if (first + 256 * j < a.tokens) atomicAdd(&count[key[j] & ((1 << DB) - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < 1 << DB; d += 256) {
    s.counts[(int64_t)d * s.blocks + blockIdx.x] = count[d];
    for (int r = 1; r < s.rounds; ++r) s.counts[(((int64_t)r << DB) + d) * s.blocks + blockIdx.x] = 0;
  }
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
template <typename T, int DB, int IPT, bool DIRECT>
__global__ __launch_bounds__(256) void sort_move_kernel(EmbedBwdArgs a, SortArgs s) {
  constexpr int D = 1 << DB, PER = D / 256;
  __shared__ uint32_t count[4][D], waves[4];
  if (blockIdx.x >= s.blocks) {
    fill<T, 256>(a, blockIdx.x - s.blocks, gridDim.x - s.blocks, s.round + 1, s.rounds + 1);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < 4 * D; i += 256) count[i / D][i % D] = 0;
  const int64_t first = (int64_t)blockIdx.x * (256 * IPT) + wave * (64 * IPT) + lane;
  uint32_t key[IPT], place[IPT], rank[IPT];
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int64_t i = first + 64 * j;
    const bool in = i < a.tokens;
    key[j] = !in ? kNoKey : s.round ? s.keys[i] : key_of(a, i);
    place[j] = !in ? 0 : s.round ? s.places[i] : (uint32_t)i;
  }
  // a thread's PER digits: tokens with the digit, and those of the blocks before
  uint32_t total[PER], before[PER], sum = 0;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const uint32_t* const c = s.counts + (int64_t)(tid * PER + q) * s.blocks;
    if constexpr (DIRECT) {
      total[q] = before[q] = 0;
#pragma unroll 8
      for (uint32_t b = 0; b < s.blocks; ++b) {
        const uint32_t n = c[b];
        total[q] += n;
        before[q] += b < blockIdx.x ? n : 0;
      }
    } else {
      total[q] = s.totals[tid * PER + q];
      before[q] = c[blockIdx.x];
    }
    sum += total[q];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < IPT; ++j) rank[j] = rank_digit<DB>((key[j] >> s.shift) & (D - 1), count[wave], lane);
  // where each wave's first token of a digit goes: behind the lower digits, the blocks and the waves before
  uint32_t lower = exclusive_sum<256>(sum, waves, tid);  // (its barriers stand behind the ranks)
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    uint32_t at = lower + before[q];
    lower += total[q];
    for (int w = 0; w < 4; ++w) {
      const uint32_t c = count[w][tid * PER + q];
      count[w][tid * PER + q] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    if (first + 64 * j >= a.tokens) continue;
    const uint32_t to = count[wave][(key[j] >> s.shift) & (D - 1)] + rank[j];
    s.keys_out[to] = key[j];
    s.places_out[to] = place[j];
    if (s.next) atomicAdd(&s.next[(int64_t)((key[j] >> (s.shift + DB)) & (D - 1)) * s.blocks + to / (256 * IPT)], 1u);
  }
}

// ------------------------------------------------------------------- sums --
struct SumArgs {
  const uint32_t* keys;
  const uint32_t* places;
  float* partial;  // [chunks, 2, ldp]: the sum of a chunk's first row, begun before it, and of its last one, which goes on
  int64_t ldp;
  int32_t chunk;   // tokens of a chunk
  int32_t chunks, g, columns;  // 1 << g threads own a vector of columns each; groups side by side over the columns
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
  const uint32_t after = i1 < a.tokens ? s.keys[i1] : kNoKey;
  uint32_t cur = s.keys[i0];
  bool begun = i0 > 0 && s.keys[i0 - 1] == cur;  // before this chunk
  float* const partial = s.partial + chunk * 2 * s.ldp + c;
  float acc[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
  uint32_t key[U], place[U];  // of the next U tokens
  auto ask = [&](int64_t i) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = min(i + u, i1 - 1);
      key[u] = s.keys[at];
      place[u] = s.places[at];
    }
  };
  ask(i0);
  for (int64_t i = i0; i < i1; i += U) {
    uint32_t now[U];
    Vec<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      now[u] = key[u];
      // (tokens that add to no row are not read)
      v[u].load(static_cast<const T*>(a.dy) + (int64_t)place[u] * a.ldy + c, key[u] < a.rows ? n : 0);
    }
    if (i + U < i1) ask(i + U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= i1) break;
      if (now[u] != cur) {
        if (begun) {
#pragma unroll
          for (int e = 0; e < VE; ++e) partial[e] = acc[e];
        } else {
          write_row<T>(a, cur, c, acc);
        }
        cur = now[u];
        begun = false;
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
      }
      if (cur >= a.rows) return;  // (these come last)
      float x[VE];
      v[u].get(x);
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[e] += x[e];
    }
  }
  if (!begun && after != cur) {
    write_row<T>(a, cur, c, acc);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) partial[(begun ? 0 : s.ldp) + e] = acc[e];
  }
}

// A block: the row that goes on from one chunk into the next ones, for one group
// of columns.  Its threads' groups take every NG-th chunk.
template <typename T>
__global__ __launch_bounds__(256) void run_join_kernel(EmbedBwdArgs a, SumArgs s) {
  constexpr int VE = kVec<T>;
  __shared__ float part[256][VE + 1];
  const int64_t chunk = blockIdx.x / s.columns, i0 = chunk * s.chunk, i1 = i0 + s.chunk;
  if (i1 >= a.tokens) return;
  const uint32_t key = s.keys[i1 - 1];
  if (key >= a.rows || s.keys[i1] != key || (i0 > 0 && s.keys[i0 - 1] == key && s.keys[i0] == key)) return;
  const int lane = threadIdx.x & ((1 << s.g) - 1), group = threadIdx.x >> s.g, groups = 256 >> s.g;
  const int c = (((int)(blockIdx.x % s.columns) << s.g) + lane) * VE;
  float acc[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
  if (c < a.cols) {
    if (group == 0) {
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[e] = s.partial[(chunk * 2 + 1) * s.ldp + c + e];
    }
    // the next B chunks' first keys and sums are asked for together
    constexpr int B = 8;
    bool more = true;
    for (int64_t b0 = chunk + 1 + group; more; b0 += (int64_t)B * groups) {
      bool goes[B];
      f32x4 v[B][VE / 4];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const int64_t b = min(b0 + (int64_t)u * groups, (int64_t)s.chunks - 1);
        goes[u] = b0 + (int64_t)u * groups < s.chunks && s.keys[b * s.chunk] == key;
#pragma unroll
        for (int q = 0; q < VE / 4; ++q)
          v[u][q] = *reinterpret_cast<const f32x4*>(s.partial + b * 2 * s.ldp + c + 4 * q);
      }
#pragma unroll
      for (int u = 0; u < B; ++u) {
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] += goes[u] ? v[u][e / 4][e % 4] : 0.0f;
      }
      more = goes[B - 1];
    }
  }
#pragma unroll
  for (int e = 0; e < VE; ++e) part[threadIdx.x][e] = acc[e];
  __syncthreads();
  if (group > 0 || c >= a.cols) return;
  for (int q = 1; q < groups; ++q) {
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[e] += part[(q << s.g) + lane][e];
  }
  write_row<T>(a, key, c, acc);
}

// ------------------------------------------------------------------- host --
constexpr int64_t kSortOne = 4096;  // tokens that one workgroup sorts

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// How a gradient is laid out over launches, and its workspace.
struct BwdPlan {
  int bits, digit, rounds;  // of the keys, of a digit, digits
  int items;                // tokens a thread of the long sort
  uint32_t blocks;          // of tokens in it
  SumArgs sum;
  size_t keys, counts, totals, partial, bytes;  // byte offsets
};
BwdPlan plan(int prec, int64_t tokens, int64_t rows, int32_t cols) {
  BwdPlan p{};
  const int ve = prec == PACK_PREC_BF16 ? 8 : 4;
  while (p.bits < 32 && (rows >> p.bits) > 0) ++p.bits;  // keys 0 .. rows
  const bool one = tokens <= kSortOne;
  p.items = tokens <= 256 * (int64_t)kDirect ? 1 : 4;
  p.blocks = one ? 0 : (uint32_t)((tokens + 256 * p.items - 1) / (256 * p.items));
  // digits of 8 bits, or of 11 where that saves a round
  p.digit = p.items > 1 && (p.bits + 10) / 11 < (p.bits + 7) / 8 ? 11 : 8;
  p.rounds = (p.bits + p.digit - 1) / p.digit;
  const int64_t vectors = ((int64_t)cols + ve - 1) / ve;
  while (p.sum.g < 6 && ((int64_t)1 << p.sum.g) < vectors) ++p.sum.g;
  p.sum.columns = (int)((vectors + (1 << p.sum.g) - 1) >> p.sum.g);
  // chunks for some 4096 waves, of 16 to 1024 tokens
  int64_t chunk = 16;
  while (chunk < 1024 && tokens * p.sum.columns * (1 << p.sum.g) / 64 > 4096 * chunk) chunk *= 2;
  p.sum.chunk = (int)chunk;
  p.sum.chunks = (int)((tokens + chunk - 1) / chunk);
  p.sum.ldp = vectors * ve;
  p.keys = 0;
  size_t at = (size_t)up(tokens * 4, 16) * (one ? 2 : 4);
  p.counts = at;
  at += (size_t)up(((int64_t)p.blocks << p.digit) * p.rounds * 4, 16);
  p.totals = at;
  at += one ? 0 : ((size_t)4 << p.digit);
  p.partial = at;
  if (p.sum.chunks > 1) at += (size_t)p.sum.chunks * 2 * (size_t)p.sum.ldp * 4;
  p.bytes = at;
  return p;
}

template <typename T, int DB, int IPT>
hipError_t sort_long(const EmbedBwdArgs& a, const BwdPlan& p, SortArgs s, uint32_t* (&buf)[2][2], uint32_t zeros,
                     hipStream_t st) {
  const dim3 grid(p.blocks + zeros), block(256);
  uint32_t* const counts = s.counts;
  s.rounds = p.rounds;
  hipLaunchKernelGGL((sort_count_kernel<T, DB, IPT>), grid, block, 0, st, a, s);
  for (int r = 0; r < p.rounds; ++r) {
    s.round = r, s.shift = r * DB;
    s.keys = buf[(r + 1) & 1][0], s.places = buf[(r + 1) & 1][1];
    s.keys_out = buf[r & 1][0], s.places_out = buf[r & 1][1];
    s.counts = counts + (((int64_t)r << DB) * p.blocks);
    s.next = r + 1 < p.rounds ? counts + (((int64_t)(r + 1) << DB) * p.blocks) : nullptr;
    if (p.blocks <= kDirect) {
      hipLaunchKernelGGL((sort_move_kernel<T, DB, IPT, true>), grid, block, 0, st, a, s);
    } else if constexpr (IPT > 1) {
      hipLaunchKernelGGL(sort_scan_kernel, dim3(1 << DB), block, 0, st, s);
      hipLaunchKernelGGL((sort_move_kernel<T, DB, IPT, false>), grid, block, 0, st, a, s);
    }
  }
  return hipGetLastError();
}

template <typename T>
hipError_t embed_bwd_t(int prec, const EmbedBwdArgs& a, hipStream_t st) {
  const BwdPlan p = plan(prec, a.tokens, a.rows, a.cols);
  if ((int64_t)p.sum.chunks * p.sum.columns >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;  // (2^32 threads)
  char* const w = static_cast<char*>(a.work);
  const int64_t list = up(a.tokens * 4, 16);
  uint32_t* buf[2][2];
  for (int i = 0; i < 4; ++i) buf[i / 2][i % 2] = reinterpret_cast<uint32_t*>(w + p.keys + i * list);
  // blocks that write zeros beside the sort: 16 KB each a launch or more, up to four a CU
  const int64_t bytes = a.rows * a.cols * (int64_t)sizeof(T);
  hipError_t e;
  int last = 0;  // the buffer that holds the sorted list
  if (a.tokens <= kSortOne) {
    const dim3 grid(1 + (uint32_t)std::min<int64_t>((bytes + 65535) / 65536, 512)), block(1024);
    if (a.tokens <= 1024)
      hipLaunchKernelGGL((sort_one_kernel<T, 1>), grid, block, 0, st, a, buf[0][0], buf[0][1], p.bits);
    else
      hipLaunchKernelGGL((sort_one_kernel<T, 4>), grid, block, 0, st, a, buf[0][0], buf[0][1], p.bits);
    e = hipGetLastError();
  } else {
    const uint32_t zeros = (uint32_t)std::min<int64_t>((bytes / (p.rounds + 1) + 16383) / 16384, 1024);
    SortArgs s{};
    s.counts = reinterpret_cast<uint32_t*>(w + p.counts), s.totals = reinterpret_cast<uint32_t*>(w + p.totals);
    s.blocks = p.blocks;
    if (p.digit == 11)
      e = sort_long<T, 11, 4>(a, p, s, buf, zeros, st);
    else
      e = p.items == 1 ? sort_long<T, 8, 1>(a, p, s, buf, zeros, st) : sort_long<T, 8, 4>(a, p, s, buf, zeros, st);
    last = (p.rounds + 1) & 1;
  }
  if (e != hipSuccess || a.tokens == 0) return e;
  SumArgs s = p.sum;
  s.keys = buf[last][0], s.places = buf[last][1];
  s.partial = reinterpret_cast<float*>(w + p.partial);
  const int64_t units = (int64_t)s.chunks * s.columns, per = 256 >> s.g;
  hipLaunchKernelGGL((run_sum_kernel<T>), dim3((uint32_t)((units + per - 1) / per)), dim3(256), 0, st, a, s);
  if (s.chunks > 1) hipLaunchKernelGGL((run_join_kernel<T>), dim3((uint32_t)units), dim3(256), 0, st, a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(int prec, const EmbedArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? embed_t<__bf16>(a, s) : embed_t<float>(a, s);
}

size_t embed_bwd_bytes(int prec, int64_t tokens, int64_t rows, int32_t cols) { return plan(prec, tokens, rows, cols).bytes; }

hipError_t launch_embed_bwd(int prec, const EmbedBwdArgs& a, hipStream_t s) {
  return prec == PACK_PREC_BF16 ? embed_bwd_t<__bf16>(prec, a, s) : embed_bwd_t<float>(prec, a, s);
}

}  // namespace tabpack
