// The embedding table of a client's model: rows of the tokens, scaled, and the table's gradient.  The gradient of a word is the
// sum over the positions at which it stands, so the positions are sorted by word first (stable, so that the sum's order, and with it
// every bit of the result, is given by the tokens alone); a block then adds up a chunk of the sorted positions in registers,
// writing each word's row once, and what a word has in several chunks is joined by a last kernel.
#include <cooperative_groups.h>

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

// A block has blockDim.x columns (vectors of a row) by blockDim.y groups of kLookupRows tokens.
template <class T, bool VEC>
__global__ void __launch_bounds__(kLookupThreads) k_embed(EmbedArgs a) {
  constexpr int E = VEC ? kPerVec<T> : 1;
  const uint32_t cols = a.dim / E;
  const uint64_t first = ((uint64_t)blockIdx.x * blockDim.y + threadIdx.y) * kLookupRows;
  const T* const table = static_cast<const T*>(a.table);
  T* const out = static_cast<T*>(a.out);
  int64_t t[kLookupRows];
#pragma unroll
  for (int r = 0; r < kLookupRows; ++r) {
    t[r] = first + r < a.n ? token_at(a.tokens, a.token_bytes, first + r) : -1;
    if (t[r] >= (int64_t)a.vocab) {
      if (a.status && threadIdx.x == 0 && blockIdx.y == 0) set_status(a.status, CVLC_ERR_INVALID_ARG);
      t[r] = -1;
    }
  }
  for (uint32_t c = blockIdx.y * blockDim.x + threadIdx.x; c < cols; c += gridDim.y * blockDim.x) {
    if constexpr (VEC) {
      uint4 raw[kLookupRows] = {};
#pragma unroll
      for (int r = 0; r < kLookupRows; ++r)
        if (t[r] >= 0) raw[r] = __ldg(reinterpret_cast<const uint4*>(table + (uint64_t)t[r] * a.table_stride) + c);
#pragma unroll
      for (int r = 0; r < kLookupRows; ++r) {
        if (first + r >= a.n) break;
        float f[E];
        if (t[r] >= 0) {
          widen<T>(raw[r], f);
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] *= a.scale;
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = 0.f;
        }
        __stcs(reinterpret_cast<uint4*>(out + (first + r) * a.out_stride) + c, narrow<T>(f));
      }
    } else {
#pragma unroll
      for (int r = 0; r < kLookupRows; ++r)
        if (first + r < a.n)
          out[(first + r) * a.out_stride + c] = from_float<T>(t[r] >= 0 ? to_float(table[(uint64_t)t[r] * a.table_stride + c]) * a.scale : 0.f);
    }
  }
}

// ---- the gradient: positions sorted by word ------------------------------------------------------
//
// Workspace: [0] status | [256] uint64[n] (word << 32 | position) | uint64[n] | float[chunks][2][dim] pieces of words at a chunk's ends
constexpr int kTokenThreads = 1024;
constexpr int kTokenWarps = kTokenThreads / 32;
constexpr int kTokenDigits = 512;
constexpr size_t kTokenShared = (size_t)kTokenWarps * kTokenDigits * 4;

CVLC_HD inline size_t eg_off_a() { return 256; }
CVLC_HD inline size_t eg_off_b(uint64_t n) { return align256(eg_off_a() + n * 8); }
CVLC_HD inline size_t eg_off_pieces(uint64_t n) { return align256(eg_off_b(n) + n * 8); }

// Positions of a chunk
constexpr uint32_t kChunkMost = 512;
uint32_t chunk_of(uint64_t n) {
  uint64_t c = 16;
  while (c < kChunkMost && (n + c - 1) / c > 2048) c *= 2;
  return (uint32_t)c;
}

// Stable radix sort by digits of up to nine bits, by one cluster.  Every warp has a stretch of the positions, in order; it counts its
// digits, the counts are scanned over warps and blocks for every digit, and the warp walks its stretch again, giving each position its
// place.  Tokens that stand for nothing (below zero, or outside the table) sort behind all words as word `vocab`.
// The other clusters of the launch, if any, write the table's zeros meanwhile.
__global__ void __launch_bounds__(kTokenThreads, 1) k_token_sort(EmbedGradArgs a, uint32_t bits, uint32_t passes, uint32_t blocks) {
  extern __shared__ uint32_t counts[];  // [warp][digit]
  __shared__ uint32_t totals[kMaxClusterBlocks][kTokenDigits];
  __shared__ uint32_t scan[kTokenWarps];
  cg::cluster_group cluster = cg::this_cluster();
  if (blockIdx.x >= blocks) {
    const uint64_t first = (uint64_t)(blockIdx.x - blocks) * kTokenThreads + threadIdx.x, stride = (uint64_t)(gridDim.x - blocks) * kTokenThreads;
    if (a.update_stride == a.dim && (reinterpret_cast<uintptr_t>(a.update) & 15) == 0) {
      zero_fill(a.update, a.vocab * a.dim, first, stride);
    } else {
      for (uint64_t i = first; i < a.vocab * a.dim; i += stride) a.update[i / a.dim * a.update_stride + i % a.dim] = 0.f;
    }
    return;
  }
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = blockIdx.x;
  int32_t* const status = static_cast<int32_t*>(a.ws);
  if (rank == 0 && tid == 0) *status = 0;
  if (blocks > 1) cluster.sync();
  else __syncthreads();
  const uint64_t stretch = ((a.n + (uint64_t)blocks * kTokenThreads - 1) / ((uint64_t)blocks * kTokenThreads)) * 32;
  const uint64_t begin = ((uint64_t)rank * kTokenWarps + warp) * stretch;
  const uint64_t end = begin + stretch < a.n ? begin + stretch : a.n;
  unsigned long long* const buf[2] = {reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a()),
                                      reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_b(a.n))};
  uint32_t* const mine = counts + warp * kTokenDigits;
  const uint32_t per = (bits + passes - 1) / passes, mask = (1u << per) - 1;
  // the first pass reads the tokens, the last one writes the first buffer
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t shift = 32 + pass * per;
    unsigned long long* const to = buf[(passes - 1 - pass) & 1];
    const unsigned long long* const from = buf[(passes - pass) & 1];
    auto item = [&](uint64_t i) -> unsigned long long {
      if (pass) return __ldcg(from + i);
      const int64_t t = token_at(a.tokens, a.token_bytes, i);
      if (t >= (int64_t)a.vocab) set_status(status, CVLC_ERR_INVALID_ARG);
      return ((unsigned long long)(t >= 0 && t < (int64_t)a.vocab ? (uint32_t)t : (uint32_t)a.vocab) << 32) | (uint32_t)i;
    };
    // lanes with the same digit
    auto peers_of = [&](uint32_t digit, uint32_t active) {
      uint32_t m = active;
      for (uint32_t b = 0; b < per; ++b) {
        const uint32_t v = __ballot_sync(kFull, (digit >> b) & 1);
        m &= (digit >> b) & 1 ? v : ~v;
      }
      return m;
    };
    for (uint32_t d = lane; d < kTokenDigits; d += 32) mine[d] = 0;
    __syncwarp();
    for (uint64_t base = begin; base < end; base += 32) {
      const bool in = base + lane < end;
      const uint32_t active = __ballot_sync(kFull, in);
      const uint32_t digit = in ? (uint32_t)(item(base + lane) >> shift) & mask : 0;
      const uint32_t peers = peers_of(digit, active);
      if (in && lane == (uint32_t)__ffs(peers) - 1) mine[digit] += __popc(peers);
      __syncwarp();
    }
    __syncthreads();
    for (uint32_t d = tid; d < kTokenDigits; d += kTokenThreads) {  // over the block's warps
      uint32_t sum = 0;
      for (int w = 0; w < kTokenWarps; ++w) {
        const uint32_t c = counts[w * kTokenDigits + d];
        counts[w * kTokenDigits + d] = sum;
        sum += c;
      }
      for (uint32_t r = 0; r < blocks; ++r) (blocks > 1 ? cluster.map_shared_rank(totals[rank], r) : totals[rank])[d] = sum;
    }
    if (blocks > 1) cluster.sync();
    else __syncthreads();
    {  // over the digits, then over the blocks before this one
      uint32_t sum = 0, before = 0;
      if (tid < kTokenDigits)
        for (uint32_t r = 0; r < blocks; ++r) {
          if (r < rank) before += totals[r][tid];
          sum += totals[r][tid];
        }
      uint32_t inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(kFull, inc, o);
        if (lane >= (uint32_t)o) inc += v;
      }
      if (lane == 31) scan[warp] = inc;
      __syncthreads();
      if (warp == 0) {
        uint32_t s = scan[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(kFull, s, o);
          if (lane >= (uint32_t)o) s += v;
        }
        scan[lane] = s;
      }
      __syncthreads();
      if (tid < kTokenDigits) {
        const uint32_t at = inc - sum + (warp ? scan[warp - 1] : 0) + before;
        for (int w = 0; w < kTokenWarps; ++w) counts[w * kTokenDigits + tid] += at;
      }
      __syncthreads();
    }
    for (uint64_t base = begin; base < end; base += 32) {
      const bool in = base + lane < end;
      const uint32_t active = __ballot_sync(kFull, in);
      const unsigned long long it = in ? item(base + lane) : 0;
      const uint32_t digit = in ? (uint32_t)(it >> shift) & mask : 0;
      const uint32_t peers = peers_of(digit, active);
      const uint32_t place = in ? mine[digit] : 0;
      __syncwarp();
      if (in) {
        to[place + __popc(peers & ((1u << lane) - 1))] = it;
        if (lane == (uint32_t)__ffs(peers) - 1) mine[digit] = place + __popc(peers);
      }
      __syncwarp();
    }
    if (blocks > 1) cluster.sync();
    else __syncthreads();
  }
}

// ---- the gradient: sums ------------------------------------------------------------------------------
constexpr int kSumThreads = 128;
constexpr int kSumAhead = 8;  // rows whose loads a thread has in flight

struct Sorted {
  const unsigned long long* at;
  uint64_t n;
  uint32_t vocab;
  // word at a place of the sorted positions; `vocab` beyond them
  __device__ __forceinline__ uint32_t word(uint64_t i) const { return i < n ? (uint32_t)(__ldg(at + i) >> 32) : vocab; }
};

template <int E>
__device__ __forceinline__ void put_row(const EmbedGradArgs& a, uint32_t word, uint32_t col, const float (&acc)[E]) {
  float* const u = a.update + (uint64_t)word * a.update_stride + (uint64_t)col * E;
  if constexpr (E == 1) {
    u[0] = a.accumulate ? u[0] + a.scale * acc[0] : a.scale * acc[0];
  } else {
#pragma unroll
    for (int q = 0; q < E / 4; ++q) {
      float4* const p = reinterpret_cast<float4*>(u) + q;
      float4 v = make_float4(a.scale * acc[4 * q], a.scale * acc[4 * q + 1], a.scale * acc[4 * q + 2], a.scale * acc[4 * q + 3]);
      if (a.accumulate) {
        const float4 o = *p;
        v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
      }
      *p = v;
    }
  }
}

// Block (chunk, slice of the columns).  A word whose positions all lie in the chunk gets its row; the piece of one that began in an
// earlier chunk goes to the chunk's first place in `pieces`, that of one that begins here and goes on to the second.
template <class T, bool VEC>
__global__ void __launch_bounds__(kSumThreads) k_embed_sum(EmbedGradArgs a, uint32_t chunk, float* pieces) {
  constexpr int E = VEC ? kPerVec<T> : 1;
  __shared__ uint32_t words[kChunkMost], where[kChunkMost];
  pdl_enter();
  const Sorted S = {reinterpret_cast<const unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a()), a.n, (uint32_t)a.vocab};
  const uint64_t first = (uint64_t)blockIdx.x * chunk;
  for (uint32_t i = threadIdx.x; i < chunk; i += kSumThreads) {
    const unsigned long long it = first + i < a.n ? __ldg(S.at + first + i) : (unsigned long long)a.vocab << 32;
    words[i] = (uint32_t)(it >> 32);
    where[i] = (uint32_t)it;
  }
  const uint32_t before = first ? S.word(first - 1) : S.vocab, after = S.word(first + chunk);
  __syncthreads();
  const uint32_t cols = a.dim / E, col = blockIdx.y * kSumThreads + threadIdx.x;
  if (col >= cols || words[0] == S.vocab) return;
  const T* const grad = static_cast<const T*>(a.grad) + (uint64_t)col * E;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  bool begun_before = before == words[0];
  for (uint32_t i = 0; i < chunk; i += kSumAhead) {
    float f[kSumAhead][E];
    if constexpr (VEC) {
      uint4 raw[kSumAhead] = {};
#pragma unroll
      for (int r = 0; r < kSumAhead; ++r)
        if (words[i + r] != S.vocab) raw[r] = __ldcs(reinterpret_cast<const uint4*>(grad + (uint64_t)where[i + r] * a.grad_stride));
#pragma unroll
      for (int r = 0; r < kSumAhead; ++r) widen<T>(raw[r], f[r]);
    } else {
#pragma unroll
      for (int r = 0; r < kSumAhead; ++r) f[r][0] = words[i + r] == S.vocab ? 0.f : to_float(grad[(uint64_t)where[i + r] * a.grad_stride]);
    }
#pragma unroll
    for (int r = 0; r < kSumAhead; ++r) {
      const uint32_t w = words[i + r];
      if (w == S.vocab) return;  // behind the last word
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += f[r][e];
      const bool last = i + r + 1 == chunk;
      const uint32_t next = last ? after : words[i + r + 1];
      if (next == w && !last) continue;
      if (begun_before || next == w) {
        float* const p = pieces + ((uint64_t)blockIdx.x * 2 + (begun_before ? 0 : 1)) * a.dim + (uint64_t)col * E;
#pragma unroll
        for (int e = 0; e < E; ++e) p[e] = acc[e];
      } else {
        put_row<E>(a, w, col, acc);
      }
      begun_before = false;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
    }
  }
}

// The word that begins in a chunk and goes on behind it: its pieces, in order
template <int E>
__global__ void __launch_bounds__(kSumThreads) k_embed_join(EmbedGradArgs a, uint32_t chunk, const float* pieces) {
  pdl_enter();
  const Sorted S = {reinterpret_cast<const unsigned long long*>(static_cast<unsigned char*>(a.ws) + eg_off_a()), a.n, (uint32_t)a.vocab};
  const uint64_t c = blockIdx.x, first = c * chunk, next = first + chunk;
  const uint32_t w = S.word(next - 1);
  if (w == S.vocab || S.word(next) != w) return;
  if (first && S.word(first - 1) == w) return;  // it began earlier
  const uint32_t col = blockIdx.y * kSumThreads + threadIdx.x;
  if (col >= a.dim / E) return;
  uint64_t lo = next, hi = a.n;  // the first place behind the word
  while (lo < hi) {
    const uint64_t mid = lo + (hi - lo) / 2;
    if (S.word(mid) == w) lo = mid + 1;
    else hi = mid;
  }
  const uint64_t last = (lo - 1) / chunk;
  float acc[E];
  const float* p = pieces + (c * 2 + 1) * a.dim + (uint64_t)col * E;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = p[e];
  for (uint64_t o = c + 1; o <= last; ++o) {
    p = pieces + o * 2 * a.dim + (uint64_t)col * E;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += p[e];
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
  const uint64_t gx = (a.n + rows - 1) / rows;
  uint64_t gy = (cols + x - 1) / x;
  if (gy > 65535) gy = 65535;
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
  const dim3 grid((unsigned)chunks, (a.dim / E + kSumThreads - 1) / kSumThreads);
  void (*const sum)(EmbedGradArgs, uint32_t, float*) = vec ? k_embed_sum<T, true> : k_embed_sum<T, false>;
  void (*const join)(EmbedGradArgs, uint32_t, const float*) = vec ? k_embed_join<kPerVec<T>> : k_embed_join<1>;
  launch_kernel(kKEmbedSum, sum, grid, dim3(kSumThreads), 0, st, true, a, chunk, pieces);
  launch_kernel(kKEmbedJoin, join, grid, dim3(kSumThreads), 0, st, true, a, chunk, pieces);
  return cudaGetLastError();
}

cudaError_t launch_token_sort(const EmbedGradArgs& a, cudaStream_t st) {
  uint32_t bits = 1;
  while ((a.vocab >> bits) != 0) ++bits;  // words 0 .. vocab
  const uint32_t passes = (bits + 8) / 9;
  const uint32_t blocks = a.n <= 2 * kTokenThreads ? 1 : kMaxClusterBlocks;
  const cudaError_t allowed = allow_shared(k_token_sort, kTokenShared);
  if (allowed != cudaSuccess) return allowed;
  LaunchScope ls(kKTokenSort, st);
  cudaLaunchConfig_t cfg = {};
  const uint32_t fill = a.accumulate ? 0 : (fill_grid(a.vocab * a.dim, 4 * kTokenThreads, kNumSM) + blocks - 1) / blocks * blocks;
  cfg.gridDim = dim3(blocks + fill);
  cfg.blockDim = dim3(kTokenThreads);
  cfg.dynamicSmemBytes = kTokenShared;
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
  const uint32_t chunk = chunk_of(n);
  return align256(eg_off_pieces(n) + (n + chunk - 1) / chunk * 2 * dim * 4);
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
