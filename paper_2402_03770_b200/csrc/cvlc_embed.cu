// The embedding table of a client's model: rows of the tokens, scaled, and the table's gradient.  The gradient of a word is the
// sum over the positions at which it stands, so the positions are sorted by word first (stable, so that the sum's order, and with it
// every bit of the result, is given by the tokens alone); a block then adds up a chunk of the sorted positions in registers,
// writing each word's row once, and what a word has in several chunks is joined by a last kernel.
#include <cooperative_groups.h>

#include <algorithm>

#include "cvlc_vocab.cuh"

namespace cg = cooperative_groups;

namespace cvlc {

namespace {

__device__ __forceinline__ int64_t token_at(const void* tokens, uint32_t token_bytes, uint64_t i) {
  return token_bytes == 8 ? static_cast<const int64_t*>(tokens)[i] : (int64_t)static_cast<const int32_t*>(tokens)[i];
}

// ---- lookup --------------------------------------------------------------------------------
constexpr int kLookupThreads = 256;
constexpr int kLookupRows = 4;  // tokens of a thread: that many independent loads

// A block has blockDim.x columns (vectors of a row) by blockDim.y groups of kLookupRows tokens, and goes from groups to groups: the next ones'
// tokens are on their way while this one's rows are.  The rows' reads bound it, or the launch: 300 x 768 32-bit values 8 us a call, 30000 rows
// of 128 bytes 6 us, in a graph.  (A block for every group, which has to wait for its tokens first: 32768 rows of 8 KB 80 us, this form 76.)
template <class T, bool VEC>
__global__ void __launch_bounds__(kLookupThreads, 6) k_embed(EmbedArgs a) {
  constexpr int E = VEC ? kPerVec<T> : 1;
  constexpr uint32_t kPadding = 0xFFFFFFFFu;
  const uint32_t cols = a.dim / E;
  const T* const table = static_cast<const T*>(a.table);
  const uint64_t step = (uint64_t)gridDim.x * blockDim.y * kLookupRows;
  uint64_t first = ((uint64_t)blockIdx.x * blockDim.y + threadIdx.y) * kLookupRows;
  bool outside = false;
  uint32_t word[kLookupRows], next[kLookupRows];
  const auto fetch = [&](uint64_t from, uint32_t (&w)[kLookupRows]) {
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
      const int64_t t = from + r < a.n ? token_at(a.tokens, a.token_bytes, from + r) : -1;
      w[r] = t >= 0 && t < (int64_t)a.vocab ? (uint32_t)t : kPadding;
      outside |= t >= (int64_t)a.vocab;
    }
  };
  fetch(first, word);
  for (; first < a.n; first += step) {
    fetch(first + step, next);
    T* const out = static_cast<T*>(a.out) + first * a.out_stride;
    const uint32_t rows = (uint32_t)min((uint64_t)kLookupRows, a.n - first);
    for (uint32_t c = blockIdx.y * blockDim.x + threadIdx.x; c < cols; c += gridDim.y * blockDim.x) {
      if constexpr (VEC) {
        uint4 raw[kLookupRows];
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
          raw[r] = make_uint4(0, 0, 0, 0);
          if (word[r] != kPadding) raw[r] = __ldg(reinterpret_cast<const uint4*>(table + word[r] * a.table_stride) + c);
        }
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
          if (r >= rows) break;
          float f[E];
          widen<T>(raw[r], f);
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = word[r] != kPadding ? f[e] * a.scale : 0.f;
          __stcs(reinterpret_cast<uint4*>(out + r * a.out_stride) + c, narrow<T>(f));
        }
      } else {
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r)
          if (r < rows) out[r * a.out_stride + c] = from_float<T>(word[r] != kPadding ? to_float(table[word[r] * a.table_stride + c]) * a.scale : 0.f);
      }
    }
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) word[r] = next[r];
  }
  if (outside && a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
}

// Long rows, of 128 vectors or more: a warp for a row, kLookupWide vectors of a lane on their way, and the next row's token.  Memory bounds it: 32768
// rows of 8 KB (24000 of them different) 71 us, 79% of the copy bandwidth, k_embed 76.  Few rows are bound by the rounds of their one warp: in a
// graph, one row of 8 KB 2.2 us (16-bit) and one of 32 KB 4.4, where the shortest rows take 1.7.
constexpr int kLookupWide = 8;
template <class T>
__global__ void __launch_bounds__(kLookupThreads, 4) k_embed_wide(EmbedArgs a) {
  constexpr int E = kPerVec<T>;
  const uint32_t cols = a.dim / E, lane = threadIdx.x & 31;
  const uint64_t step = (uint64_t)gridDim.x * (kLookupThreads / 32);
  uint64_t row = (uint64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5);
  int64_t next = row < a.n ? token_at(a.tokens, a.token_bytes, row) : -1;
  for (; row < a.n; row += step) {
    const int64_t word = next;
    next = row + step < a.n ? token_at(a.tokens, a.token_bytes, row + step) : -1;
    const bool there = word >= 0 && word < (int64_t)a.vocab;
    if (word >= (int64_t)a.vocab && a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
    const uint4* const from = reinterpret_cast<const uint4*>(static_cast<const T*>(a.table) + (there ? (uint64_t)word : 0) * a.table_stride);
    uint4* const to = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + row * a.out_stride);
    for (uint32_t c = lane; c < cols; c += 32 * kLookupWide) {
      uint4 raw[kLookupWide];
#pragma unroll
      for (int j = 0; j < kLookupWide; ++j) {
        raw[j] = make_uint4(0, 0, 0, 0);
        if (there && c + 32 * j < cols) raw[j] = __ldg(from + c + 32 * j);
      }
#pragma unroll
      for (int j = 0; j < kLookupWide; ++j) {
        if (c + 32 * j >= cols) break;
        float f[E];
        widen<T>(raw[j], f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = there ? f[e] * a.scale : 0.f;
        __stcs(to + c + 32 * j, narrow<T>(f));
      }
    }
  }
}

// ---- the gradient: positions sorted by word ------------------------------------------------------
//
// Workspace: [0] status | [256] uint64[n] (word << 32 | position) | uint64[n] | float[chunks_most][2][dim] pieces of words at a chunk's ends
constexpr int kTokenThreads = 1024;
constexpr int kTokenWarps = kTokenThreads / 32;
constexpr int kTokenDigits = 512;
constexpr size_t kTokenShared = (size_t)kTokenWarps * kTokenDigits * 4;
constexpr int kSortAhead = 4;  // loads of a thread in flight

CVLC_HD inline size_t eg_off_a() { return 256; }
CVLC_HD inline size_t eg_off_b(uint64_t n) { return align256(eg_off_a() + n * 8); }
CVLC_HD inline size_t eg_off_pieces(uint64_t n) { return align256(eg_off_b(n) + n * 8); }

// Positions of a chunk
constexpr uint32_t kChunkLeast = 16, kChunkMost = 512, kChunksWanted = 2048;
uint32_t chunk_of(uint64_t n) {
  uint64_t c = kChunkLeast;
  while (c < kChunkMost && (n + c - 1) / c > kChunksWanted) c *= 2;
  return (uint32_t)c;
}
// The most chunks that n positions or fewer have: a longer chunk is taken from some number of positions on, and a workspace
// serves every call that is not larger than the one that it was made for.
uint64_t chunks_most(uint64_t n) {
  return std::max(std::min<uint64_t>((n + kChunkLeast - 1) / kChunkLeast, kChunksWanted), (n + kChunkMost - 1) / kChunkMost);
}

// What the sort's launch does besides, where the table is written out: zeros for the rows of words that do not occur.  The blocks have the
// rows in turn (the words that occur are often the first ones); a block looks through all tokens for those of its rows, unless they are so
// many that writing zeros to all rows is less.
constexpr uint64_t kMarkedTokens = 1u << 18;
__device__ __forceinline__ void zero_absent(const EmbedGradArgs& a, uint32_t block, uint32_t blocks, uint32_t* marks, uint32_t mark_words) {
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, vocab = (uint32_t)a.vocab;
  if (block >= vocab) return;
  const uint32_t rows = (vocab - 1 - block) / blocks + 1;  // row i of the block: block + i * blocks
  const bool marked = a.n <= kMarkedTokens && rows <= mark_words * 32;
  if (marked) {
    for (uint32_t i = tid; i < (rows + 31) / 32; i += blockDim.x) marks[i] = 0;
    __syncthreads();
    for (uint64_t i = tid; i < a.n; i += 8 * kTokenThreads) {
      int64_t t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = i + j * kTokenThreads < a.n ? token_at(a.tokens, a.token_bytes, i + j * kTokenThreads) : -1;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (t[j] < 0 || t[j] >= (int64_t)vocab) continue;
        const uint32_t row = (uint32_t)t[j] / blocks;
        if ((uint32_t)t[j] - row * blocks == block) atomicOr(&marks[row >> 5], 1u << (row & 31));
      }
    }
    __syncthreads();
  }
  const bool vec = a.dim % 4 == 0 && a.update_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.update) & 15) == 0;
  for (uint32_t r = warp; r < rows; r += kTokenWarps) {
    if (marked && (marks[r >> 5] >> (r & 31) & 1)) continue;
    float* const u = a.update + ((uint64_t)r * blocks + block) * a.update_stride;
    if (vec) {
      for (uint32_t c = lane; c < a.dim / 4; c += 32) __stcs(reinterpret_cast<float4*>(u) + c, make_float4(0.f, 0.f, 0.f, 0.f));
    } else {
      for (uint32_t c = lane; c < a.dim; c += 32) u[c] = 0.f;
    }
  }
}

// word << 32 | position; a token that stands for nothing is word `vocab`
__device__ __forceinline__ unsigned long long sort_item(const EmbedGradArgs& a, uint64_t i, bool& outside) {
  const int64_t t = token_at(a.tokens, a.token_bytes, i);
  outside |= t >= (int64_t)a.vocab;
  return ((unsigned long long)(t >= 0 && t < (int64_t)a.vocab ? (uint32_t)t : (uint32_t)a.vocab) << 32) | (uint32_t)i;
}
// the lanes of `active` with this lane's digit of `bits` bits
__device__ __forceinline__ uint32_t peers_of(uint32_t digit, uint32_t bits, uint32_t active) {
  uint32_t m = active;
#pragma unroll
  for (uint32_t b = 0; b < 9; ++b) {
    if (b >= bits) break;
    const uint32_t own = 0u - ((digit >> b) & 1u);
    m &= ~(__ballot_sync(kFull, own) ^ own);
  }
  return m;
}
// Exclusive scan over the first 2^n threads' values, n at most 10, by a block of 1024 threads
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* scan) {
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(kFull, inc, o);
    if (lane >= (uint32_t)o) inc += u;
  }
  if (lane == 31) scan[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    uint32_t s = scan[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(kFull, s, o);
      if (lane >= (uint32_t)o) s += u;
    }
    scan[lane] = s;
  }
  __syncthreads();
  return inc - v + (warp ? scan[warp - 1] : 0);
}

// A warp's next 32 items to their places: what the digits before, the blocks, groups and warps before have (`base`, `mine`), and the lanes before
__device__ __forceinline__ void place_items(unsigned long long it, bool in, uint32_t shift, uint32_t bits, uint32_t* mine, const uint32_t* base,
                                            unsigned long long* to) {
  const uint32_t lane = threadIdx.x & 31, digit = (uint32_t)(it >> shift) & ((1u << bits) - 1);
  const uint32_t peers = peers_of(digit, bits, __ballot_sync(kFull, in));
  const uint32_t place = in ? mine[digit] : 0;
  __syncwarp();
  if (in) {
    to[base[digit] + place + __popc(peers & ((1u << lane) - 1))] = it;
    if (lane == (uint32_t)__ffs(peers) - 1) mine[digit] = place + __popc(peers);
  }
  __syncwarp();
}

// Up to 2048 positions: one block holds them, in registers while they are counted and in shared memory from pass to pass.  (The cluster
// needs two of its barriers a pass, with everything written to memory behind each; but with 8192 positions one block takes twice its time.)
constexpr int kBlockItems = 2;
constexpr uint64_t kBlockSort = (uint64_t)kBlockItems * kTokenThreads;
template <int ITEMS>
__device__ void sort_in_block(const EmbedGradArgs& a, uint32_t bits, uint32_t passes, uint32_t* counts, unsigned long long* held, uint32_t* group_base,
                              uint32_t* scan) {
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = (uint32_t)a.n;
  int32_t* const status = static_cast<int32_t*>(a.ws);
  if (tid == 0) *status = 0;
  __syncthreads();
  const uint32_t begin = warp * ITEMS * 32;
  const uint32_t per = (bits + passes - 1) / passes, digits = 1u << per, mask = digits - 1;
  const uint32_t groups = kTokenThreads / digits < kTokenWarps ? kTokenThreads / digits : kTokenWarps, group_warps = kTokenWarps / groups;
  uint32_t* const mine = counts + warp * digits;
  unsigned long long it[ITEMS];
  bool outside = false;
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) it[j] = begin + 32 * j + lane < n ? sort_item(a, begin + 32 * j + lane, outside) : 0;
  if (outside) set_status(status, CVLC_ERR_INVALID_ARG);
  unsigned long long* const out = reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a());
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t shift = 32 + pass * per;
    for (uint32_t d = lane; d < digits; d += 32) mine[d] = 0;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
      if (begin + 32 * j + lane < n) atomicAdd(&mine[(uint32_t)(it[j] >> shift) & mask], 1u);
    __syncthreads();
    if (tid < groups * digits) {  // over a group's warps
      const uint32_t d = tid & mask, first = tid / digits * group_warps;
      uint32_t sum = 0;
      for (uint32_t w = first; w < first + group_warps; ++w) {
        const uint32_t c = counts[w * digits + d];
        counts[w * digits + d] = sum;
        sum += c;
      }
      group_base[tid] = sum;
    }
    __syncthreads();
    uint32_t sum = 0;
    if (tid < digits)
      for (uint32_t g = 0; g < groups; ++g) {
        const uint32_t c = group_base[g * digits + tid];
        group_base[g * digits + tid] = sum;
        sum += c;
      }
    const uint32_t at = block_scan(sum, scan);
    if (tid < digits)
      for (uint32_t g = 0; g < groups; ++g) group_base[g * digits + tid] += at;
    __syncthreads();
    const bool last = pass + 1 == passes;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) place_items(it[j], begin + 32 * j + lane < n, shift, per, mine, group_base + warp / group_warps * digits, last ? out : held);
    if (last) break;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
      if (begin + 32 * j + lane < n) it[j] = held[begin + 32 * j + lane];
    __syncthreads();
  }
}

// Stable radix sort by digits of up to nine bits, by one cluster.  What bounds it is its chain of passes, each of two walks and two cluster
// barriers, on eight SMs: 8192 tokens of 32000 words 18 us with the launch.  The zeros of the launch's other blocks hide it where the table is
// large (65537 tokens beside 512 MB of table: 88 us, which 112 blocks take for 345 MB of zeros; being clusters as well, they leave 28
// SMs without a block, and a plain fill of all 512 MB takes 76).  Clusters of 4 leave the zeros more SMs and the sort
// fewer: 17308 tokens beside 22 MB 31 us for the whole gradient, with 8 27; beside 512 MB 180 and 180.  Every warp has a stretch of the positions, in order; it counts its
// digits (in any order), the counts are scanned over warps (in groups, side by side) and blocks for every digit, and the warp walks its stretch again, giving
// each position its place.  Tokens that stand for nothing (below zero, or outside the table) sort behind all words as word `vocab`.
__global__ void __launch_bounds__(kTokenThreads, 1) k_token_sort(EmbedGradArgs a, uint32_t bits, uint32_t passes, uint32_t blocks) {
  extern __shared__ uint32_t counts[];  // [warp][digit]
  __shared__ uint32_t totals[kMaxClusterBlocks][kTokenDigits];
  __shared__ uint32_t group_base[kTokenThreads];  // [group][digit]
  __shared__ uint32_t scan[kTokenWarps];
  cg::cluster_group cluster = cg::this_cluster();
  if (blocks == 1 && blockIdx.x == 0) {
    unsigned long long* const held = reinterpret_cast<unsigned long long*>(counts + kTokenWarps * kTokenDigits);
    sort_in_block<kBlockItems>(a, bits, passes, counts, held, group_base, scan);
    return;
  }
  if (blockIdx.x >= blocks) {
    zero_absent(a, blockIdx.x - blocks, gridDim.x - blocks, counts, kTokenShared / 4);
    return;
  }
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = blockIdx.x;
  int32_t* const status = static_cast<int32_t*>(a.ws);
  if (rank == 0 && tid == 0) *status = 0;
  cluster.sync();
  const uint64_t stretch = ((uint32_t)a.n / (blocks * kTokenThreads) + 1) * 32;
  const uint64_t begin = ((uint64_t)rank * kTokenWarps + warp) * stretch;
  const uint64_t end = begin + stretch < a.n ? begin + stretch : a.n;
  unsigned long long* const buf[2] = {reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a()),
                                      reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_b(a.n))};
  const uint32_t per = (bits + passes - 1) / passes, digits = 1u << per, mask = digits - 1;
  // groups of warps whose counts of a digit one thread adds up: 1024 threads, a digit and a group each
  const uint32_t groups = kTokenThreads / digits < kTokenWarps ? kTokenThreads / digits : kTokenWarps, group_warps = kTokenWarps / groups;
  uint32_t* const mine = counts + warp * digits;
  const uint32_t* const my_base = group_base + warp / group_warps * digits;
  // the first pass reads the tokens, the last one writes the first buffer
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t shift = 32 + pass * per;
    unsigned long long* const to = buf[(passes - 1 - pass) & 1];
    const unsigned long long* const from = buf[(passes - pass) & 1];
    bool outside = false;
    auto item = [&](uint64_t i) { return pass ? __ldcg(from + i) : sort_item(a, i, outside); };
    for (uint32_t d = lane; d < digits; d += 32) mine[d] = 0;
    __syncwarp();
    for (uint64_t base = begin; base < end; base += 32 * kSortAhead) {
      unsigned long long it[kSortAhead];
#pragma unroll
      for (int j = 0; j < kSortAhead; ++j) it[j] = base + 32 * j + lane < end ? item(base + 32 * j + lane) : 0;
#pragma unroll
      for (int j = 0; j < kSortAhead; ++j)
        if (base + 32 * j + lane < end) atomicAdd(&mine[(uint32_t)(it[j] >> shift) & mask], 1u);
    }
    if (outside) set_status(status, CVLC_ERR_INVALID_ARG);
    __syncthreads();
    for (uint32_t i = tid; i < groups * digits; i += kTokenThreads) {  // over a group's warps
      const uint32_t d = i & mask, first = i / digits * group_warps;
      uint32_t sum = 0;
      for (uint32_t w = first; w < first + group_warps; ++w) {
        const uint32_t c = counts[w * digits + d];
        counts[w * digits + d] = sum;
        sum += c;
      }
      group_base[i] = sum;
    }
    __syncthreads();
    if (tid < digits) {  // over the groups
      uint32_t sum = 0;
      for (uint32_t g = 0; g < groups; ++g) {
        const uint32_t c = group_base[g * digits + tid];
        group_base[g * digits + tid] = sum;
        sum += c;
      }
      for (uint32_t r = 0; r < blocks; ++r) cluster.map_shared_rank(totals[rank], r)[tid] = sum;
    }
    cluster.sync();
    {  // over the digits, then over the blocks before this one
      uint32_t sum = 0, before = 0;
      if (tid < digits)
        for (uint32_t r = 0; r < blocks; ++r) {
          if (r < rank) before += totals[r][tid];
          sum += totals[r][tid];
        }
      const uint32_t at = block_scan(sum, scan) + before;
      if (tid < digits) {
        for (uint32_t g = 0; g < groups; ++g) group_base[g * digits + tid] += at;
      }
      __syncthreads();
    }
    for (uint64_t base = begin; base < end; base += 32 * kSortAhead) {
      unsigned long long it[kSortAhead];
#pragma unroll
      for (int j = 0; j < kSortAhead; ++j) it[j] = base + 32 * j + lane < end ? item(base + 32 * j + lane) : 0;
#pragma unroll
      for (int j = 0; j < kSortAhead; ++j) {
        if (base + 32 * j >= end) break;
        place_items(it[j], base + 32 * j + lane < end, shift, per, mine, my_base, to);
      }
    }
    cluster.sync();
  }
}

// ---- the gradient: sums ------------------------------------------------------------------------------
constexpr int kSumThreads = 128;
constexpr uint32_t kSumPlaces = 1024;  // positions of a block
constexpr int kSumAhead = 8;   // rows whose loads a thread has in flight
constexpr int kJoinAhead = 8;  // and pieces

struct Sorted {
  const unsigned long long* at;
  uint64_t n;
  uint32_t vocab;
  // word at a place of the sorted positions; `vocab` beyond them
  __device__ __forceinline__ uint32_t word(uint64_t i) const { return i < n ? (uint32_t)(__ldg(at + i) >> 32) : vocab; }
};

// A word's row, or a part of it.  Added by reductions in memory, which nothing waits for: a row is added to once in a kernel, so they
// have no order (8192 rows of 4 KB added: 17 us, reading the rows first 22).  They take subnormal numbers for 0.
template <int E>
__device__ __forceinline__ void put_row(const EmbedGradArgs& a, uint32_t word, uint32_t col, const float (&acc)[E]) {
  float* const u = a.update + (uint64_t)word * a.update_stride + (uint64_t)col * E;
  if constexpr (E == 1) {
    if (a.accumulate) atomicAdd(u, a.scale * acc[0]);
    else u[0] = a.scale * acc[0];
  } else {
#pragma unroll
    for (int q = 0; q < E; q += 4) {
      const float4 v = make_float4(a.scale * acc[q], a.scale * acc[q + 1], a.scale * acc[q + 2], a.scale * acc[q + 3]);
      if (a.accumulate) asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(u + q), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
      else __stcs(reinterpret_cast<float4*>(u + q), v);
    }
  }
}

template <int E>
__device__ __forceinline__ void put_piece(float* p, const float (&v)[E]) {
  if constexpr (E == 1) {
    p[0] = v[0];
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
  }
}
template <int E>
__device__ __forceinline__ void get_piece(const float* p, float (&v)[E]) {
  if constexpr (E == 1) {
    v[0] = p[0];
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 q = *reinterpret_cast<const float4*>(p + e);
      v[e] = q.x, v[e + 1] = q.y, v[e + 2] = q.z, v[e + 3] = q.w;
    }
  }
}

// Block (chunks, slice of the columns): kSumThreads / `width` chunks, `width` columns, so that short rows leave no thread idle (100000 rows of 64 32-bit
// values, the whole gradient: 60 us with a chunk a block, 54 so).  Memory bounds it: 65537 rows of 4 KB 87 us, 8192 rows of 2 KB, added,
// 17.  A word whose positions all lie in the chunk gets its row;
// the piece of one that began in an earlier chunk goes to the chunk's first place in `pieces`, that of one that begins here and goes
// on to the second.
template <class T, bool VEC>
__global__ void __launch_bounds__(kSumThreads) k_embed_sum(EmbedGradArgs a, uint32_t chunk, uint32_t width, float* pieces) {
  constexpr int E = VEC ? kPerVec<T> : 1;
  __shared__ uint32_t words_of[kSumPlaces], where_of[kSumPlaces];
  pdl_enter();
  const Sorted S = {reinterpret_cast<const unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a()), a.n, (uint32_t)a.vocab};
  const uint32_t here = kSumThreads / width, mine = threadIdx.x / width;
  for (uint32_t i = threadIdx.x; i < here * chunk; i += kSumThreads) {
    const uint64_t at = (uint64_t)blockIdx.x * here * chunk + i;
    const unsigned long long it = at < a.n ? __ldg(S.at + at) : (unsigned long long)a.vocab << 32;
    words_of[i] = (uint32_t)(it >> 32);
    where_of[i] = (uint32_t)it;
  }
  const uint64_t c = (uint64_t)blockIdx.x * here + mine, first = c * chunk;
  const uint32_t *const words = words_of + mine * chunk, *const where = where_of + mine * chunk;
  const uint32_t before = first ? S.word(first - 1) : S.vocab, after = S.word(first + chunk);
  __syncthreads();
  const uint32_t cols = a.dim / E, col = blockIdx.y * width + threadIdx.x % width;
  if (col >= cols || words[0] == S.vocab) return;
  const T* const grad = static_cast<const T*>(a.grad) + (uint64_t)col * E;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  bool begun_before = before == words[0];
  for (uint32_t i = 0; i < chunk; i += kSumAhead) {
    uint4 raw[VEC ? kSumAhead : 1] = {};
    float one[VEC ? 1 : kSumAhead];
#pragma unroll
    for (int r = 0; r < kSumAhead; ++r) {
      const T* const from = grad + (uint64_t)where[i + r] * a.grad_stride;
      if constexpr (VEC) {
        if (words[i + r] != S.vocab) raw[r] = __ldcs(reinterpret_cast<const uint4*>(from));
      } else {
        one[r] = words[i + r] == S.vocab ? 0.f : to_float(*from);
      }
    }
#pragma unroll
    for (int r = 0; r < kSumAhead; ++r) {
      const uint32_t w = words[i + r];
      if (w == S.vocab) return;  // behind the last word
      if constexpr (VEC) {
        float f[E];
        widen<T>(raw[r], f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += f[e];
      } else {
        acc[0] += one[r];
      }
      const bool last = i + r + 1 == chunk;
      const uint32_t next = last ? after : words[i + r + 1];
      if (next == w && !last) continue;
      if (begun_before || next == w) {
        put_piece<E>(pieces + (c * 2 + (begun_before ? 0 : 1)) * a.dim + (uint64_t)col * E, acc);
      } else {
        put_row<E>(a, w, col, acc);
      }
      begun_before = false;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
    }
  }
}

// The word that begins in a chunk and goes on behind it: its pieces, in order.  Latency bounds it: the launch, and the chain of a word that has many
// chunks (8192 tokens 8.6 us, 65537 13).  Four groups of threads for a quarter of the pieces each make every block large, and the blocks of
// the words that do not go on cost more than the chains save (65537 x 2048: 181 us for the whole gradient, so 172; 26336 positions of 616 words
// 87 and 68).
template <int E>
__global__ void __launch_bounds__(kSumThreads) k_embed_join(EmbedGradArgs a, uint32_t chunk, const float* pieces) {
  pdl_enter();
  const Sorted S = {reinterpret_cast<const unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a()), a.n, (uint32_t)a.vocab};
  const uint64_t c = blockIdx.x, first = c * chunk, next = first + chunk;
  const uint32_t w = S.word(next - 1);
  if (w == S.vocab || S.word(next) != w) return;
  if (first && S.word(first - 1) == w) return;  // it began earlier
  const uint32_t col = blockIdx.y * kSumThreads + threadIdx.x;
  uint64_t last = c + 1;  // the last chunk that begins with the word, 32 chunks at a time
  for (;; last += 32) {
    const uint32_t more = __ballot_sync(kFull, S.word((last + 1 + (threadIdx.x & 31)) * chunk) == w);
    if (more != kFull) {
      last += __ffs(~more) - 1;
      break;
    }
  }
  if (col >= a.dim / E) return;
  float acc[E];
  get_piece<E>(pieces + (c * 2 + 1) * a.dim + (uint64_t)col * E, acc);
  for (uint64_t o = c + 1; o <= last; o += kJoinAhead) {
    float f[kJoinAhead][E];
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j) get_piece<E>(pieces + (o + j <= last ? o + j : last) * 2 * a.dim + (uint64_t)col * E, f[j]);
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j)
      if (o + j <= last)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += f[j][e];
  }
  put_row<E>(a, w, col, acc);
}

template <class T>
cudaError_t embed_typed(const EmbedArgs& a, cudaStream_t st) {
  const uintptr_t bits = reinterpret_cast<uintptr_t>(a.table) | reinterpret_cast<uintptr_t>(a.out);
  const bool vec = (bits & 15) == 0 && a.dim % kPerVec<T> == 0 && a.table_stride % kPerVec<T> == 0 && a.out_stride % kPerVec<T> == 0;
  const uint32_t cols = vec ? a.dim / kPerVec<T> : a.dim;
  uint32_t x = 32;
  while (x < kLookupThreads && x < cols) x *= 2;
  const dim3 block(x, kLookupThreads / x);
  const uint64_t rows = (uint64_t)block.y * kLookupRows;
  const uint64_t resident = 6 * kNumSM;
  const uint64_t gy = std::min<uint64_t>((cols + x - 1) / x, resident);
  const uint64_t gx = std::min((a.n + rows - 1) / rows, (resident + gy - 1) / gy);
  if (vec && cols >= 128) {
    const uint64_t blocks = (a.n + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
    launch_kernel(kKEmbed, k_embed_wide<T>, dim3((unsigned)std::min<uint64_t>(blocks, 4 * kNumSM)), dim3(kLookupThreads), 0, st, false, a);
    return cudaGetLastError();
  }
  void (*const kernel)(EmbedArgs) = vec ? k_embed<T, true> : k_embed<T, false>;
  launch_kernel(kKEmbed, kernel, dim3((unsigned)gx, (unsigned)gy), block, 0, st, false, a);
  return cudaGetLastError();
}

template <class T>
cudaError_t embed_grad_typed(const EmbedGradArgs& a, cudaStream_t st) {
  const uint32_t chunk = chunk_of(a.n);
  const uint64_t chunks = (a.n + chunk - 1) / chunk;
  float* const pieces = reinterpret_cast<float*>(static_cast<unsigned char*>(a.ws) + eg_off_pieces(a.n));
  const bool vec = (reinterpret_cast<uintptr_t>(a.grad) & 15) == 0 && (reinterpret_cast<uintptr_t>(a.update) & 15) == 0 &&
                   a.dim % kPerVec<T> == 0 && a.grad_stride % kPerVec<T> == 0 && a.update_stride % 4 == 0;
  const uint32_t E = vec ? kPerVec<T> : 1;
  const uint32_t cols = a.dim / E;
  uint32_t width = kSumThreads;  // columns of a block; short rows leave room for several chunks
  while (width > 4 && width / 2 >= cols && kSumThreads / (width / 2) * chunk <= kSumPlaces) width /= 2;
  const uint32_t here = kSumThreads / width;
  void (*const sum)(EmbedGradArgs, uint32_t, uint32_t, float*) = vec ? k_embed_sum<T, true> : k_embed_sum<T, false>;
  void (*const join)(EmbedGradArgs, uint32_t, const float*) = vec ? k_embed_join<kPerVec<T>> : k_embed_join<1>;
  launch_kernel(kKEmbedSum, sum, dim3((unsigned)((chunks + here - 1) / here), (cols + width - 1) / width), dim3(kSumThreads), 0, st, true, a, chunk, width,
                pieces);
  launch_kernel(kKEmbedJoin, join, dim3((unsigned)chunks, (cols + kSumThreads - 1) / kSumThreads), dim3(kSumThreads), 0, st, true, a, chunk, pieces);
  return cudaGetLastError();
}

// clusters of the sort that the current device runs at once, asked for once per device
uint32_t clusters_at_once() {
  static OncePerDevice once;
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 2;
  const cudaError_t e = once_per_device(once, [&] {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kMaxClusterBlocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kMaxClusterBlocks);
    cfg.blockDim = dim3(kTokenThreads);
    cfg.dynamicSmemBytes = kTokenShared;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    const cudaError_t r = cudaOccupancyMaxActiveClusters(&n, k_token_sort, &cfg);
    if (r == cudaSuccess) known[dev].store(n < 2 ? 2 : n, std::memory_order_relaxed);
    return r;
  });
  return e == cudaSuccess ? (uint32_t)known[dev].load(std::memory_order_relaxed) : 2;
}

cudaError_t launch_token_sort(const EmbedGradArgs& a, cudaStream_t st) {
  uint32_t bits = 1;
  while ((a.vocab >> bits) != 0) ++bits;  // words 0 .. vocab
  const uint32_t passes = (bits + 8) / 9;
  const uint32_t blocks = a.n <= kBlockSort ? 1 : kMaxClusterBlocks;
  const size_t smem = kTokenShared + (blocks == 1 ? (a.n < kTokenThreads ? kTokenThreads : a.n) * 8 : 0);
  static OncePerDevice once;
  const cudaError_t allowed = once_per_device(once, [] { return allow_shared(k_token_sort, kTokenShared + kBlockSort * 8); });
  if (allowed != cudaSuccess) return allowed;
  LaunchScope ls(kKTokenSort, st);
  cudaLaunchConfig_t cfg = {};
  // blocks beside those of the sort that write zeros: as many whole clusters as run at once, since a second round of them would double the time
  uint32_t fill = 0;
  if (!a.accumulate) {
    fill = fill_grid(a.vocab * a.dim, 4 * kTokenThreads, kNumSM - 1);
    if (blocks > 1) {
      const uint32_t most = (clusters_at_once() - 1) * blocks;
      fill = std::min((fill + blocks - 1) / blocks * blocks, most);
    }
  }
  cfg.gridDim = dim3(blocks + fill);
  cfg.blockDim = dim3(kTokenThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = blocks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = blocks > 1 ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_token_sort, a, bits, passes, blocks);
  const cudaError_t last = cudaGetLastError();
  return e != cudaSuccess ? e : last;
}

}  // namespace

size_t embed_grad_ws_bytes(uint64_t n, uint32_t dim) {
  return align256(eg_off_pieces(n) + chunks_most(n) * 2 * dim * 4);
}

cudaError_t launch_embed(const EmbedArgs& a, uint32_t dtype, cudaStream_t st) {
  if (dtype == CVLC_F32) return embed_typed<float>(a, st);
  if (dtype == CVLC_F16) return embed_typed<__half>(a, st);
  return embed_typed<__nv_bfloat16>(a, st);
}

cudaError_t launch_embed_grad(const EmbedGradArgs& a, uint32_t dtype, cudaStream_t st) {
  const cudaError_t e = launch_token_sort(a, st);
  if (e != cudaSuccess || a.n == 0) return e;
  if (dtype == CVLC_F32) return embed_grad_typed<float>(a, st);
  if (dtype == CVLC_F16) return embed_grad_typed<__half>(a, st);
  return embed_grad_typed<__nv_bfloat16>(a, st);
}

}  // namespace cvlc
