// Softmax cross entropy of hidden states against a head matrix, and its gradients, without holding the logits, but where they are few.
//
// z_tv = scale h_t . w_v;  loss_t = weight_t (ln sum_v exp(z_tv) - z_t,target);  G_tv = weight_t (q_tv - [v = target]);
// dh_t = scale sum_v G_tv w_v;  dw_v = scale sum_t G_tv h_t
//
// Three products of rows x vocab x dim each.  The first one's values never leave the tensor memory: a tile of them becomes, per row, its maximum
// and its sum of exponentials (k_head_stats), which are joined to the row's loss and ln sum exp (k_head_rows).  For the gradients a piece of the
// vocabulary at a time is multiplied again and becomes G, rounded to the type of the operands (k_head_probs), from which come the piece of the head's
// gradient (k_head_grad) and the piece's part of the hidden states' (k_head_parts, in fp32, joined by k_head_join).  In one piece the exponentials are kept
// (k_head_keep); few logits are kept themselves (k_head_logits, k_head_softmax).
#include <math.h>

#include "cvlc_tensor.cuh"
#include "cvlc_vocab.cuh"

namespace cvlc {

bool make_tensor_map(CUtensorMap* map, const void* base, bool bf16, uint64_t cols, uint64_t rows, uint64_t stride, uint32_t box_cols, uint32_t box_rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static std::atomic<void*> found{nullptr};
  void* at = found.load(std::memory_order_acquire);
  if (!at) {
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &at, 12000, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess)
      return false;
    found.store(at, std::memory_order_release);
  }
  const cuuint64_t size[2] = {cols, rows}, apart[1] = {stride * 2};
  const cuuint32_t box[2] = {box_cols, box_rows}, step[2] = {1, 1};
  return reinterpret_cast<Encode>(at)(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(base), size, apart,
                                      box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The kernel behind may be set up while this one runs: the small ones fit beside a block of the products, and a block of theirs moves in as soon as an
// SM is free; it waits for the rest before it reads or writes anything that this one does.  The rule: a kernel first waits for the one in front (pdl_enter()), then lets
// the next one in.  So when a kernel starts, all kernels of the call but the one directly in front are complete, and so is what the caller has in front of the call, whose
// first kernel is an ordinary launch.  What they have written, and the one in front does not write, may be read ahead of the wait (`early`).
__device__ __forceinline__ void let_next_in() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- the products --------------------------------------------------------------------------
// A block has a tile of 128 rows by 256 columns, a pair of blocks one of 256 by 256: one thread copies operands (a ring of stages of 64 values of the
// sum), one issues the products, eight warps read a finished tile from the tensor memory while the next one is made in its other half.
constexpr uint32_t kTileM = 128, kTileN = 256, kTileK = 64;
constexpr int kThreads = 384, kOutWarps = 8;
constexpr uint32_t kBoxBytes = 32 * 128;  // of a warp, 32 rows of 64 columns on their way out
// The ring's stages hold 64 values of the sum of a block's rows and columns.  A pair has six of 32 KB.  A block of its own with few rows copies only those: the
// products read what follows them as rows, too, which nobody looks at, and there is room for more stages (8 x 4096 x 131072: 207 -> 171 us, the copy bandwidth).
constexpr uint32_t kRingBytes = 192 * 1024;
constexpr int kMostStages = 8;
constexpr uint32_t kPairBytes = (kTileM + kTileN / 2) * kTileK * 2, kPairStages = kRingBytes / kPairBytes;
constexpr size_t kGemmShared = kRingBytes + kOutWarps * kBoxBytes + 1024;

struct Header {  // at the beginning of the workspace
  float up, down;         // fp16: a power of two that brings weights to at most 1, times 2^15, and its inverse
  uint32_t wild;          // some row is
  uint32_t late[kNumSM];  // a block of the products has given up
};
__device__ __forceinline__ bool any_late(const Header* h) {  // asked by all threads of a block
  uint32_t x = 0;
  for (uint32_t i = threadIdx.x; i < kNumSM; i += blockDim.x) x |= h->late[i];
  return __syncthreads_or((int)x) != 0;
}

enum Epilogue { kStats, kKeep, kKeepOwn, kKeepWide, kProbs, kParts, kGrad, kBoth };  // kBoth: parts, then grad
struct Product {
  CUtensorMap a, b, c;                   // c: the output, where it is of 16 bits and its rows lie on 16 bytes
  uint32_t m, n, k_blocks;               // rows, columns, steps of 64 of the sum
  uint32_t tile_n, tiles_m, tiles_n, splits;  // columns of a tile; splits of the sum
  uint32_t a_bytes, b_bytes, stage_bytes, stages;  // of the ring
  uint32_t values;                       // of the sum in a stage: 64, or what there is if that is less and both operands come rows first
  uint32_t m_first, group;               // tiles of one column of tiles follow one another, else those of a row; so many of them, then the next column
  uint32_t col0, token_bytes;            // stats, probs: the word of column 0
  float k2, alpha;                       // scale log2(e); factor of the output
  const void* targets;
  float2* stats;                         // (maximum, sum relative to it) of a row's half tile
  float* at_target;                      // z of the row's target, in log2
  uint64_t stats_stride;
  const float4* row;                     // probs: what makes a row's G of its z
  void* out;
  uint64_t ldo, split_stride;
  uint32_t add, wide;                    // added to what is there; written by boxes
  uint32_t whole;                        // both: a gradient itself, not a part of it
  const float* alpha_dev;                // or nullptr; multiplies alpha
  const uint32_t* skip;                  // or nullptr; where it is 0 nothing is to be done
  const uint32_t* wild;                  // or nullptr; of 256 rows each: 0 where they are left out
  Header* header;
  int32_t* status;
  uint32_t first;                        // of the call's products
  uint32_t early;                        // the operands are there before the kernel in front has ended
  uint32_t lost_copy, lost_tile;         // self-test: the tiles of a block from which on nothing is copied, its readers give up
  uint64_t most;                         // nanoseconds, of every wait
};
template <int EPI>
struct Products {
  static constexpr int count = EPI == kBoth ? 2 : 1;
  Product p[count];
};
__device__ __forceinline__ void tile_of(const Product& g, uint32_t t, uint32_t* tm, uint32_t* tn) {
  const uint32_t fast = g.m_first ? g.tiles_m : g.tiles_n, slow = g.m_first ? g.tiles_n : g.tiles_m;
  const uint32_t first = t / (g.group * slow) * g.group, here = min(g.group, fast - first), r = t - first * slow;
  const uint32_t i = first + r % here, j = r / here;
  *tm = g.m_first ? i : j, *tn = g.m_first ? j : i;
}
__device__ __forceinline__ bool left_out(const Product& g, uint32_t w) {
  if (!g.wild) return false;
  uint32_t tm, tn;
  tile_of(g, w % (g.tiles_m * g.tiles_n), &tm, &tn);
  return g.wild[tm] == 0;  // a pair's tile, or the only one
}

struct Work {
  uint32_t m0, n0, n_end, slot, k_from, k_to, split;
};
template <int CG>
__device__ __forceinline__ Work work_of(const Product& g, uint32_t w) {
  const uint32_t tiles = g.tiles_m * g.tiles_n, split = w / tiles, t = w - split * tiles;
  uint32_t tm, tn;
  tile_of(g, t, &tm, &tn);
  Work r;
  r.m0 = (tm * CG + pair_rank<CG>()) * kTileM, r.n0 = tn * g.tile_n, r.n_end = min(g.n, r.n0 + g.tile_n), r.slot = 2 * tn, r.split = split;
  r.k_from = (uint32_t)((uint64_t)g.k_blocks * split / g.splits), r.k_to = (uint32_t)((uint64_t)g.k_blocks * (split + 1) / g.splits);
  return r;
}

template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
  }
}
__device__ __forceinline__ int64_t target_of(const void* targets, uint32_t bytes, uint64_t row) {
  return bytes == 8 ? static_cast<const int64_t*>(targets)[row] : static_cast<const int32_t*>(targets)[row];
}

// 64 columns of a thread's row, in 16 bits, by way of shared memory: lines of 128 bytes go out whole, and nothing is left to do but start the copy.
// (Threads that store their rows themselves, 32 bytes at a time, take as long; they leave four times as many requests.)
__device__ __forceinline__ void row_to_box(uint32_t box, uint32_t lane, uint32_t part, const uint32_t (&p)[16]) {
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + lane * 128 + ((4 * part + i) ^ (lane & 7)) * 16), "r"(p[4 * i]), "r"(p[4 * i + 1]),
                 "r"(p[4 * i + 2]), "r"(p[4 * i + 3])
                 : "memory");
}
__device__ __forceinline__ void box_free(uint32_t lane) {
  if (lane == 0) tiles_read();
  __syncwarp();
}
__device__ __forceinline__ void box_out(const CUtensorMap& map, uint32_t box, uint32_t lane, uint32_t x, uint32_t y) {
  shared_written();
  __syncwarp();
  if (lane == 0) store_tile(map, box, x, y);
}

// What becomes of a warp's 32 rows and 128 columns of a finished tile
template <int EPI, class T>
__device__ __forceinline__ void finish_tile(const Product& g, const Work& w, uint32_t tensor, uint32_t half, uint32_t quarter, uint32_t lane, uint32_t box) {
  const uint32_t row = w.m0 + quarter * 32 + lane;
  const bool there = row < g.m;
  float v[32];
  if constexpr (EPI == kStats) {
    const int64_t target = there ? target_of(g.targets, g.token_bytes, row) - g.col0 : -1;
    float most = -CUDART_INF_F, sum = 0.0f;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (col >= w.n_end) break;
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = v[i] * g.k2;
      if (w.n_end - col < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (col + i >= w.n_end) v[i] = -CUDART_INF_F;
      }
      const bool mine = target >= col && target < (int64_t)col + 32;
      if (__any_sync(kFull, mine)) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (mine && target == (int64_t)col + i) g.at_target[row] = v[i], v[i] = -CUDART_INF_F;
      }
      float m = v[0];
#pragma unroll
      for (int i = 1; i < 32; ++i) m = fmaxf(m, v[i]);
      m = fmaxf(m, most);
      const float from = m == -CUDART_INF_F ? 0.0f : m;
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < 32; ++i) s += exp2_fast(v[i] - from);
      sum = fmaf(sum, exp2_fast(most - from), s);
      most = m;
    }
    if (there) g.stats[(uint64_t)(w.slot + half) * g.stats_stride + row] = make_float2(most, sum);
  } else if constexpr (EPI == kKeep) {
    // relative to the target's own value, known from before: what is kept needs no second look.  A row of which some word is more than 2^60 times as likely as
    // the target is wild and gets a second turn, relative to its maximum.
    const float from = there ? g.at_target[row] : CUDART_INF_F;
    const int64_t target = there ? target_of(g.targets, g.token_bytes, row) : -1;
    const bool counts = from != CUDART_INF_F;
    float most = -CUDART_INF_F, sum = 0.0f;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if ((c & 1) == 0) {
        if (col >= w.n_end) break;
        box_free(lane);
      }
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = fmaf(v[i], g.k2, -from);
      const bool mine = target >= col && target < (int64_t)col + 32;
      if (col + 32 > w.n_end || __any_sync(kFull, mine)) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (col + i >= w.n_end || (mine && target == (int64_t)col + i)) v[i] = -CUDART_INF_F;
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) most = fmaxf(most, v[i]), v[i] = exp2_fast(v[i]);
      float s[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
      for (int i = 4; i < 32; ++i) s[i & 3] += v[i];
      sum += (s[0] + s[1]) + (s[2] + s[3]);
      uint32_t p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = counts ? pack2<T>(v[2 * i], v[2 * i + 1]) : 0u;
      row_to_box(box, lane, c & 1, p);
      if (c & 1) box_out(g.c, box, lane, col - 32, w.m0 + quarter * 32);
    }
    if (there) g.stats[(uint64_t)(w.slot + half) * g.stats_stride + row] = make_float2(most, sum);
  } else if constexpr (EPI == kKeepOwn || EPI == kKeepWide) {
    // each row of 128 columns relative to its own maximum, which takes a look of its own: in fp16, which has no range to spare, and in fp32 (wide)
    const int64_t target = there ? target_of(g.targets, g.token_bytes, row) : -1;
    // (by pairs, all 128 columns are held meanwhile)
    constexpr bool held = EPI == kKeepOwn;
    constexpr int unrolled = held ? 4 : 1;
    float z[held ? 4 : 1][32], most = -CUDART_INF_F, sum = 0.0f;
    if (held) {
#pragma unroll
      for (int c = 0; c < 4; ++c) tensor_load(tensor + c * 32, z[held ? c : 0]);
    }
#pragma unroll unrolled
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (!held && col >= w.n_end) break;
      float (&v)[32] = z[held ? c : 0];
      if (!held) tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = v[i] * g.k2;
      const bool mine = target >= col && target < (int64_t)min(col + 32, w.n_end);
      if (col + 32 > w.n_end || __any_sync(kFull, mine)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if (mine && target == (int64_t)col + i) g.at_target[row] = v[i], v[i] = -CUDART_INF_F;
          if (col + i >= w.n_end) v[i] = -CUDART_INF_F;
        }
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) most = fmaxf(most, v[i]);
    }
    const float from = most == -CUDART_INF_F ? 0.0f : most;
#pragma unroll unrolled
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (EPI == kKeepWide ? col >= w.n_end : (c & 1) == 0 && col >= w.n_end) break;
      if (EPI == kKeepOwn && (c & 1) == 0) box_free(lane);
      float (&v)[32] = z[held ? c : 0];
      if (held) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] -= from;
      } else {
        tensor_load(tensor + c * 32, v);
        tensor_loaded(v);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = fmaf(v[i], g.k2, -from);
        const bool mine = target >= col && target < (int64_t)col + 32;
        if (col + 32 > w.n_end || __any_sync(kFull, mine)) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (col + i >= w.n_end || (mine && target == (int64_t)col + i)) v[i] = -CUDART_INF_F;
        }
      }
      float s[4] = {};
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = exp2_fast(v[i]), s[i & 3] += v[i];
      sum += (s[0] + s[1]) + (s[2] + s[3]);
      if constexpr (EPI == kKeepWide) {
        float* const out = static_cast<float*>(g.out) + (uint64_t)row * g.ldo + col;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t p[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = __float_as_uint(v[8 * h + i]);
          if (there) store_sector(out + 8 * h, p);
        }
      } else {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
        row_to_box(box, lane, c & 1, p);
        if (c & 1) box_out(g.c, box, lane, col - 32, w.m0 + quarter * 32);
      }
    }
    if (there) g.stats[(uint64_t)(w.slot + half) * g.stats_stride + row] = make_float2(most, sum);
  } else if constexpr (EPI == kProbs) {
    // x: ln sum exp in log2; y: the weight, times the power of two by which G is raised, 0 where the row counts for nothing; z: the target's G
    const float4 r = there ? g.row[row] : make_float4(0, 0, 0, 0);
    const int64_t target = there ? target_of(g.targets, g.token_bytes, row) - g.col0 : -1;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if ((c & 1) == 0) {
        if (col >= w.n_end) break;
        box_free(lane);
      }
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = r.y == 0.0f ? 0.0f : exp2_fast(fmaf(v[i], g.k2, -r.x)) * r.y;
      const bool mine = target >= col && target < (int64_t)col + 32;
      if (__any_sync(kFull, mine)) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (mine && target == (int64_t)col + i) v[i] = r.z;
      }
      uint32_t p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
      row_to_box(box, lane, c & 1, p);
      if (c & 1) box_out(g.c, box, lane, col - 32, w.m0 + quarter * 32);
    }
  } else if constexpr (EPI == kParts) {
    float* const out = static_cast<float*>(g.out) + w.split * g.split_stride + (uint64_t)row * g.ldo;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (col >= w.n_end) break;
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
      if (there) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t p[8];
          if (g.add) {
            load_sector(out + col + 8 * h, p);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = __float_as_uint(__uint_as_float(p[i]) + v[8 * h + i]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = __float_as_uint(v[8 * h + i]);
          }
          store_sector(out + col + 8 * h, p);
        }
      }
    }
  } else {
    T* const out = static_cast<T*>(g.out);
    const float alpha = g.alpha_dev ? g.alpha * *g.alpha_dev : g.alpha;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if ((c & 1) == 0) {
        if (col >= w.n_end) break;
        box_free(lane);  // in either form: the tile before this one may have been the launch's other product's, on its way from this box
      }
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
      uint32_t p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = pack2<T>(v[2 * i] * alpha, v[2 * i + 1] * alpha);
      if (g.wide) {
        row_to_box(box, lane, c & 1, p);
        if (c & 1) box_out(g.c, box, lane, col - 32, w.m0 + quarter * 32);
      } else if (col < w.n_end) {  // rows that begin anywhere: turned in shared memory, so that a warp writes neighbours
#pragma unroll
        for (int i = 0; i < 16; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(box + (lane * 17 + i) * 4), "r"(p[i]) : "memory");
        __syncwarp();
        uint16_t* const to = reinterpret_cast<uint16_t*>(out) + (uint64_t)(w.m0 + quarter * 32) * g.ldo + col + lane;
        const uint32_t rows = min(32u, g.m - min(g.m, w.m0 + quarter * 32));
        if (col + lane < w.n_end)
          for (uint32_t r = 0; r < rows; ++r) {
            uint16_t x;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(box + r * 68 + lane * 2) : "memory");
            to[r * g.ldo] = x;
          }
        __syncwarp();
      }
    }
  }
}

// where a block's first n tiles end
__device__ __forceinline__ uint32_t first_tiles(uint32_t n, uint32_t first, uint32_t apart, uint32_t items) {
  return (uint32_t)min((uint64_t)items, first + (uint64_t)n * apart);
}

template <int EPI, bool A_ROWS, bool B_ROWS, class T, int CG>
__global__ void __launch_bounds__(kThreads, 1) k_head_product(const __grid_constant__ Products<EPI> both) {
  extern __shared__ uint8_t dynamic[];
  __shared__ uint64_t full[kMostStages], empty[kMostStages], made[2], taken[2], over;
  __shared__ uint32_t tensor_at, late, other_late, copies;  // late: somebody of this block has given up; of the pair's other one; stages whose copies this one has begun
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31, rank = pair_rank<CG>();
  const uint32_t ring = (smem_at(dynamic) + 1023) & ~1023u;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMostStages; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 1);
    for (int i = 0; i < 2; ++i) mbar_init(made + i, 1), mbar_init(taken + i, CG * kOutWarps);
    mbar_init(&over, 1);
    late = other_late = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tensor_alloc<CG>(&tensor_at);
  tensor_before();
  __syncthreads();
  pair_sync<CG>();
  tensor_after();
  const Product& g0 = both.p[0];
  const uint32_t stages = CG == 2 ? kPairStages : g0.stages, stage_bytes = CG == 2 ? kPairBytes : g0.stage_bytes;
  const uint32_t tensor = tensor_at, first = blockIdx.x / CG, apart = gridDim.x / CG;
  if (!g0.early || warp >= 4) {
    pdl_enter();
    let_next_in();
  }
  const uint32_t items0 = g0.skip && *g0.skip == 0 ? 0 : g0.tiles_m * g0.tiles_n * g0.splits;
  const Product& last = both.p[Products<EPI>::count - 1];
  const uint32_t items = items0 + (EPI == kBoth ? last.tiles_m * last.tiles_n * last.splits : 0);
  bool ok = true, multiplied = false;
  if (warp == 0 && lane == 0) {
    uint32_t s = 0, phase = 0, issued = 0;
    const uint32_t end = first_tiles(g0.lost_copy, first, apart, items);
    for (uint32_t w = first; ok && w < end; w += apart) {
      const bool second = EPI == kBoth && w >= items0;
      const Product& g = both.p[second ? Products<EPI>::count - 1 : 0];
      if (left_out(g, w)) continue;
      const Work r = work_of<CG>(g, second ? w - items0 : w);
      const bool a_rows = EPI == kBoth ? second : A_ROWS;
      const uint32_t a_bytes = CG == 2 ? kTileM * kTileK * 2 : g.a_bytes, bytes = CG == 2 ? 2 * kPairBytes : a_bytes + g.b_bytes, values = CG == 2 ? kTileK : g.values;
      for (uint32_t k = r.k_from; k < r.k_to; ++k) {
        if (!(ok = mbar_wait(empty + s, phase ^ 1, &late, g0.most))) break;
        if (rank == 0) mbar_expect(full + s, bytes);
        const uint32_t a = ring + s * stage_bytes, b = a + a_bytes, bar = leader_at<CG>(smem_at(full + s)), n0 = r.n0 + rank * (g.tile_n / CG);
        if (a_rows) {
#pragma unroll
          for (uint32_t i = 0; i < kTileM / 64; ++i) load_tile<CG>(g.a, a + i * values * 128, bar, r.m0 + 64 * i, k * kTileK);
        } else {
          load_tile<CG>(g.a, a, bar, k * kTileK, r.m0);
        }
        if constexpr (B_ROWS) {  // tiles of 256 columns only
#pragma unroll
          for (uint32_t i = 0; i < kTileN / CG / 64; ++i) load_tile<CG>(g.b, b + i * values * 128, bar, n0 + 64 * i, k * kTileK);
        } else {
          load_tile<CG>(g.b, b, bar, k * kTileK, n0);
        }
        ++issued;
        if (++s == stages) s = 0, phase ^= 1;
      }
    }
    copies = issued;
    // what the products report of the last stages reaches this block before it leaves
    for (uint32_t i = issued - min(issued, stages); ok && i < issued; ++i) ok = mbar_wait(empty + i % stages, i / stages & 1, &late, g0.most);
  } else if (warp == 1 && lane == 0 && rank == 0) {
    constexpr bool bf16 = std::is_same<T, __nv_bfloat16>::value;
    uint32_t s = 0, phase = 0, turn_of = 0;
    for (uint32_t w = first; ok && w < items; w += apart) {
      const bool second = EPI == kBoth && w >= items0;
      const Product& g = both.p[second ? Products<EPI>::count - 1 : 0];
      if (left_out(g, w)) continue;
      const Work r = work_of<CG>(g, second ? w - items0 : w);
      const bool a_rows = EPI == kBoth ? second : A_ROWS;
      const uint32_t kind = product_kind(bf16, a_rows, B_ROWS, CG * kTileM, g.tile_n);
      const uint32_t a_bytes = CG == 2 ? kTileM * kTileK * 2 : g.a_bytes, values = CG == 2 ? kTileK : g.values;
      const uint32_t half = turn_of & 1;
      if (!(ok = mbar_wait(taken + half, (turn_of / 2 & 1) ^ 1, &late, g0.most))) break;
      tensor_after();
      for (uint32_t k = r.k_from; k < r.k_to; ++k) {
        if (!(ok = mbar_wait(full + s, phase, &late, g0.most))) break;
        tensor_after();
        const uint32_t a = ring + s * stage_bytes, b = a + a_bytes;
#pragma unroll
        for (uint32_t i = 0; i < kTileK / 16; ++i)
          if (!B_ROWS || i * 16 < values)
            multiply<CG>(tensor + half * kTileN,
                         a_rows ? operand<true>(a + i * kStepBytes<true>, values) : operand<false>(a + i * kStepBytes<false>, values),
                         operand<B_ROWS>(b + i * kStepBytes<B_ROWS>, values), kind, k != r.k_from || i != 0);
        commit<CG>(empty + s);
        multiplied = true;
        if (++s == stages) s = 0, phase ^= 1;
      }
      if (ok) commit<CG>(made + half);
      ++turn_of;
    }
  } else if (warp >= 4) {
    const uint32_t half_tile = (warp - 4) / 4, quarter = warp & 3, box = ring + kRingBytes + (warp - 4) * kBoxBytes;
    const uint32_t end = first_tiles(g0.lost_tile, first, apart, items);
    uint32_t turn_of = 0, w = first;
    for (; w < end; w += apart) {
      const bool second = EPI == kBoth && w >= items0;
      const Product& g = both.p[second ? Products<EPI>::count - 1 : 0];
      if (left_out(g, w)) continue;
      const Work r = work_of<CG>(g, second ? w - items0 : w);
      const uint32_t half = turn_of & 1;
      if (!(ok = __all_sync(kFull, mbar_wait(made + half, turn_of / 2 & 1, &late, g0.most)))) break;
      tensor_after();
      const uint32_t at = tensor + half * kTileN + half_tile * 128 + (quarter * 32 << 16);
      if constexpr (EPI == kBoth) {
        if (g.whole) finish_tile<kGrad, T>(g, r, at, half_tile, quarter, lane, box);
        else finish_tile<kParts, T>(g, r, at, half_tile, quarter, lane, box);
      } else {
        finish_tile<EPI, T>(g, r, at, half_tile, quarter, lane, box);
      }
      tensor_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_leader<CG>(taken + half);
      ++turn_of;
    }
    if (w < items && ok) ok = false, *static_cast<volatile uint32_t*>(&late) = 1;
    if (EPI == kBoth && !ok && g0.whole)  // no kernel follows that would say it: what is missing of the hidden states' gradient is NaN
      for (; w < items0; w += apart) {
        const Work r = work_of<CG>(g0, w);
        const uint32_t row = r.m0 + quarter * 32 + lane, from = r.n0 + half_tile * 128;
        if (row < g0.m)
          for (uint32_t col = from; col < min(r.n_end, from + 128); ++col) static_cast<T*>(g0.out)[row * g0.ldo + col] = from_float<T>(CUDART_NAN_F);
      }
    if (lane == 0) tiles_stored();
  }
  __syncwarp();
  tensor_before();
  __syncthreads();
  if (CG == 2 && threadIdx.x == 0 && late) shared_store(other_at(smem_at(&other_late)), 1);
  pair_sync<CG>();
  tensor_after();
  if (late || (CG == 2 && other_late)) {  // alike for both blocks of a pair.  What they have begun ends before they leave:
    if (threadIdx.x == 0 && rank == 0) {  // the copies of the last stages, of both,
      const uint32_t others = CG == 2 ? shared_load(other_at(smem_at(&copies))) : copies, most = max(copies, others);
      for (uint32_t i = most - min(most, stages); i < most; ++i) {
        uint32_t none = 0;
        uint64_t* const b = full + i % stages;
        if (i >= copies) mbar_expect(b, kPairBytes);  // begun by the other block alone
        if (i >= others) mbar_came(b, kPairBytes);    // expected of it, and not begun
        mbar_wait(b, i / stages & 1, &none, g0.most / 4);
      }
    }
    if (multiplied) {  // and the products, where all are issued, too, and readers alone have given up
      uint32_t none = 0;
      commit<CG>(&over);
      mbar_wait(&over, 0, &none, g0.most / 4);
    }
    __syncwarp();
    tensor_before();
    pair_sync<CG>();
    tensor_after();
  }
  if (warp == 2) tensor_free<CG>(tensor);
  if (threadIdx.x == 128) {  // of the warps that have waited for the kernel in front
    for (uint32_t i = blockIdx.x; i < kNumSM; i += gridDim.x) {
      if (g0.first) g0.header->late[i] = late;  // nobody has written here
      else if (late) g0.header->late[i] = 1;
    }
    if (late && g0.status) set_status(g0.status, CVLC_ERR_DEVICE_TIMEOUT);
  }
}

// ---- what is around them -------------------------------------------------------------------

// One block, fp16 with weights only: the power of two by which G is held.  fp16 holds 2^-24 to 2^16; G, at most the largest weight in size, is held at most 2^15.
__global__ void __launch_bounds__(1024) k_head_begin(Header* h, const float* weight, const void* targets, uint32_t token_bytes, uint64_t rows, uint32_t vocab) {
  pdl_enter();
  let_next_in();
  __shared__ uint32_t most;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  uint32_t m = 0;
  for (uint64_t i = threadIdx.x; i < rows; i += blockDim.x) {
    const int64_t t = target_of(targets, token_bytes, i);
    const uint32_t w = __float_as_uint(weight[i]) & 0x7FFFFFFFu;
    if (t >= 0 && t < (int64_t)vocab && w < 0x7F800000u) m = max(m, w);
  }
  m = __reduce_max_sync(kFull, m);
  if ((threadIdx.x & 31) == 0) atomicMax(&most, m);
  __syncthreads();
  if (threadIdx.x == 0) {
    const int e = (most ? min(max((int)(most >> 23) - 126, -100), 100) : 0) - 15;
    h->up = exp2f((float)-e), h->down = exp2f((float)e);
  }
}

// Rows of any alignment, copied to rows on 16 bytes, a warp each.  Rows that count for nothing become zeros: their values, which may be no numbers, have a part
// in the products of others' gradients.
struct AlignJob {
  const uint16_t* from;
  uint16_t* to;
  uint64_t from_stride, to_stride, rows;
  const void* targets;  // or nullptr: all rows count
};
struct AlignArgs {
  AlignJob of[2];
  uint32_t blocks;  // of the first
  uint32_t dim, token_bytes, vocab;
  const float* weight;
};
__global__ void __launch_bounds__(256) k_head_align(const __grid_constant__ AlignArgs all) {
  pdl_enter();
  let_next_in();
  const bool second = blockIdx.x >= all.blocks;
  const AlignJob& a = all.of[second];
  const uint64_t row = (uint64_t)(blockIdx.x - (second ? all.blocks : 0)) * 8 + threadIdx.x / 32;
  const uint32_t lane = threadIdx.x & 31, dim = all.dim;
  if (row >= a.rows) return;
  const uint16_t* const src = a.from + row * a.from_stride;
  uint16_t* const dst = a.to + row * a.to_stride;
  bool counts = true;
  if (a.targets) {
    const int64_t t = target_of(a.targets, all.token_bytes, row);
    counts = t >= 0 && t < (int64_t)all.vocab && !(all.weight && all.weight[row] == 0.0f);
  }
  // rows that begin anywhere are read by the two vectors that hold eight elements
  const uint32_t lead = (uint32_t)(reinterpret_cast<uintptr_t>(src) % 16 / 2);
  const uint4* const vectors = reinterpret_cast<const uint4*>(src - lead);
  for (uint32_t i = lane * 8; i < dim; i += 256) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (counts) {
      if (lead == 0 ? i + 8 <= dim : i >= lead && i + 16 - lead <= dim) {
        const uint4 x = __ldg(vectors + i / 8), y = lead ? __ldg(vectors + i / 8 + 1) : x;
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        const uint32_t skip = lead / 2, bits = (lead & 1) * 16;
        uint32_t z[5];
#pragma unroll
        for (int k = 0; k < 5; ++k) z[k] = skip == 0 ? w[k] : skip == 1 ? w[k + 1] : skip == 2 ? w[k + 2] : w[k + 3 < 8 ? k + 3 : 7];
        v = make_uint4(__funnelshift_r(z[0], z[1], bits), __funnelshift_r(z[1], z[2], bits), __funnelshift_r(z[2], z[3], bits),
                       __funnelshift_r(z[3], z[4], bits));
      } else {
        uint32_t x[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) x[k] = i + k < dim ? src[i + k] : 0;
        v = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
      }
    }
    *reinterpret_cast<uint4*>(dst + i) = v;  // rows of the copy are filled up to eight
  }
}

// The target's logit as the loss is made of it.  +infinity would be a loss of 0: all others' exponentials relative to it are 0.
__device__ __forceinline__ float known(float zt) { return zt < CUDART_INF_F ? zt : CUDART_NAN_F; }

// z of every row's target, in log2; +inf where the row counts for nothing.  A warp a row.
struct TargetArgs {
  const void *hidden, *head, *targets;
  uint64_t hidden_ld, head_ld, rows;
  uint32_t dim, vocab, token_bytes, blocks_wild;
  const float* weight;
  float* at_target;
  float k2;
  uint32_t* wild;
  Header* header;
};
__global__ void __launch_bounds__(256) k_head_target(const TargetArgs a) {
  pdl_enter();
  let_next_in();
  const uint64_t row = (uint64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const uint32_t lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.header->wild = 0;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < a.blocks_wild; i += (uint64_t)gridDim.x * 256) a.wild[i] = 0;
  if (row >= a.rows) return;
  const int64_t t = target_of(a.targets, a.token_bytes, row);
  if (t < 0 || t >= (int64_t)a.vocab || (a.weight && a.weight[row] == 0.0f)) {
    if (lane == 0) a.at_target[row] = CUDART_INF_F;
    return;
  }
  const __nv_bfloat16* const h = static_cast<const __nv_bfloat16*>(a.hidden) + row * a.hidden_ld;
  const __nv_bfloat16* const w = static_cast<const __nv_bfloat16*>(a.head) + (uint64_t)t * a.head_ld;
  float sum = 0.0f;
#pragma unroll 4
  for (uint32_t i = lane * 8; i < a.dim; i += 256) {
    if (i + 8 <= a.dim) {
      float x[8], y[8];
      widen<__nv_bfloat16>(__ldg(reinterpret_cast<const uint4*>(h + i)), x);
      widen<__nv_bfloat16>(__ldg(reinterpret_cast<const uint4*>(w + i)), y);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum = fmaf(x[k], y[k], sum);
    } else {
      for (uint32_t k = i; k < a.dim; ++k) sum = fmaf(to_float(h[k]), to_float(w[k]), sum);
    }
  }
#pragma unroll
  for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(kFull, sum, d);
  sum *= a.k2;
  if (lane == 0) a.at_target[row] = known(sum);
}

constexpr float kWild = 60.0f;
constexpr uint32_t kWildRows = 2 * kTileM;  // that get a second turn together
struct RowsArgs {
  const float2* stats;
  uint64_t stats_stride;
  uint32_t slots, token_bytes, vocab;
  float* at_target;
  const void* targets;
  const float* weight;
  float* loss;
  float4* row;  // or nullptr
  Header* header;
  uint64_t rows;
  int32_t* status;
  const float* up;  // multiplies the weight, or nullptr: up_by does
  float up_by;
  // where the exponentials are kept:
  __nv_bfloat16* kept;
  uint64_t ldg, hidden_ld, scaled_ld;
  const __nv_bfloat16* hidden;
  __nv_bfloat16* scaled;  // hidden states times their rows' factor
  float *factor, *raised;  // raised: by how much a row's second reference is above its target, 0: not at all
  uint32_t* wild;
  uint32_t dim, second;
};
constexpr uint32_t kRowsOf = 8, kGroups = 32;  // rows of a block, threads of a row

// two parts of a row (maximum, sum): of sums relative to their own maxima, or of sums of the same reference
__device__ __forceinline__ float2 join_two(float2 x, float2 y, bool relative) {
  const float m = fmaxf(x.x, y.x), from = m == -CUDART_INF_F ? 0.0f : m;
  return make_float2(m, relative ? x.y * exp2f(x.x - from) + y.y * exp2f(y.x - from) : x.y + y.y);
}
// The parts of a block's rows joined: eight threads hold what is left of each, one of a warp.  Returns whether a block of the products has given up.
__device__ __forceinline__ bool join_parts(const RowsArgs& a, uint64_t row, uint32_t group, bool relative, float2 (*part)[kRowsOf]) {
  static_assert(kNumSM <= 256, "a thread for every block");
  const uint32_t late = threadIdx.x < kNumSM ? a.header->late[threadIdx.x] : 0;
  float2 sum = make_float2(-CUDART_INF_F, 0.0f);
  if (row < a.rows) {
    const float2* const from = a.stats + row;
    uint32_t i = group;
    for (; i + 3 * kGroups < a.slots; i += 4 * kGroups) {
      float2 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = from[(uint64_t)(i + k * kGroups) * a.stats_stride];
#pragma unroll
      for (int k = 0; k < 4; ++k) sum = join_two(sum, x[k], relative);
    }
    for (; i < a.slots; i += kGroups) sum = join_two(sum, from[(uint64_t)i * a.stats_stride], relative);
  }
#pragma unroll
  for (int d = kRowsOf; d < 32; d *= 2) {
    const float2 other = make_float2(__shfl_xor_sync(kFull, sum.x, d), __shfl_xor_sync(kFull, sum.y, d));
    sum = join_two(sum, other, relative);
  }
  if ((threadIdx.x & 31) < kRowsOf) part[threadIdx.x / 32][threadIdx.x % kRowsOf] = sum;
  return __syncthreads_or((int)late) != 0;
}

// A row of hidden states as it counts: others, which may hold anything, would have a part in the head's gradient
__device__ __forceinline__ void masked_row(const uint16_t* h, uint16_t* to, uint32_t dim, bool counts, uint32_t from, uint32_t threads) {
#pragma unroll 4
  for (uint32_t i = from; i < dim; i += threads * 8) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (counts) {
      if (i + 8 <= dim) {
        v = __ldg(reinterpret_cast<const uint4*>(h + i));
      } else {
        uint32_t x[8] = {};
        for (uint32_t k = 0; i + k < dim; ++k) x[k] = h[i + k];
        v = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
      }
    }
    *reinterpret_cast<uint4*>(to + i) = v;
  }
}

// A row's parts joined.  Sums relative to the largest; that of the words other than the target (o) is kept apart, so that 1 - q and a small loss
// ln(1 + o) keep their accuracy.
__global__ void __launch_bounds__(256) k_head_rows(const RowsArgs a) {
  pdl_enter();
  if (a.row) let_next_in();  // else the last of the call
  __shared__ float2 part[8][kRowsOf];
  __shared__ uint32_t counts[kRowsOf];
  const uint32_t group = threadIdx.x / kRowsOf, lane = threadIdx.x % kRowsOf;
  const uint64_t row = (uint64_t)blockIdx.x * kRowsOf + lane;
  const bool late = join_parts(a, row, group, true, part);
  if (group == 0 && row < a.rows) {
    const int64_t target = target_of(a.targets, a.token_bytes, row);
    const float weight = a.weight ? a.weight[row] : 1.0f;
    if (target >= (int64_t)a.vocab && a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
    const bool there = target >= 0 && target < (int64_t)a.vocab && weight != 0.0f;
    counts[lane] = there;
    float loss = 0.0f;
    float4 r = make_float4(0, 0, 0, 0);
    if (there) {
      const float zt = known(a.at_target[row]);
      float most = zt;
      for (uint32_t i = 0; i < 8; ++i) most = fmaxf(most, part[i][lane].x);
      double others = 0.0;
      for (uint32_t i = 0; i < 8; ++i)
        if (part[i][lane].x != -CUDART_INF_F || part[i][lane].y != 0.0f) others += (double)(part[i][lane].y * exp2f(part[i][lane].x - most));
      const float o = (float)others, right = exp2f(zt - most), total = right + o, w = weight * (a.up ? *a.up : a.up_by);
      loss = weight * (most == zt ? log1pf(o) : logf(total) + (most - zt) * kLn2);
      r = make_float4(most + log2f(total), w, -(o / total) * w, 0.0f);
    }
    a.loss[row] = late ? CUDART_NAN_F : loss;
    if (a.row) a.row[row] = r;
  }
  if (!a.scaled) return;
  __syncthreads();
  const uint64_t mine = (uint64_t)blockIdx.x * kRowsOf + threadIdx.x / 32;
  if (mine >= a.rows) return;
  masked_row(reinterpret_cast<const uint16_t*>(a.hidden) + mine * a.hidden_ld, reinterpret_cast<uint16_t*>(a.scaled) + mine * a.scaled_ld, a.dim,
             counts[threadIdx.x / 32], (threadIdx.x & 31) * 8, 32);
}

// The same where the exponentials are kept, relative to the target's (to the row's maximum in a second turn): of G = weight exp(z - from) / total the
// factor goes into the hidden states, row by row, and the target's own value, - o, to its place.
__global__ void __launch_bounds__(256) k_head_rows_kept(const RowsArgs a) {
  pdl_enter();
  let_next_in();
  __shared__ float2 part[8][kRowsOf];
  __shared__ float factors[kRowsOf];
  if (a.second && a.header->wild == 0) return;
  if (a.second && a.wild[(uint64_t)blockIdx.x * kRowsOf / kWildRows] == 0) return;
  const uint32_t group = threadIdx.x / kRowsOf, lane = threadIdx.x % kRowsOf;
  const uint64_t row = (uint64_t)blockIdx.x * kRowsOf + lane;
  const uint64_t row0 = (uint64_t)blockIdx.x * kRowsOf;
  const uint32_t warp = threadIdx.x / 32, at = (threadIdx.x & 31) * 8;
  const __nv_bfloat16* const h = a.hidden + (row0 + warp) * a.hidden_ld;
  uint4 ahead[4];  // the beginning of the hidden states, on its way meanwhile
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (row0 + warp < a.rows && at + k * 256 + 8 <= a.dim) ahead[k] = __ldg(reinterpret_cast<const uint4*>(h + at + k * 256));
  const bool late = join_parts(a, row, group, false, part);
  if (group == 0 && row < a.rows) {
    const int64_t target = target_of(a.targets, a.token_bytes, row);
    const float weight = a.weight ? a.weight[row] : 1.0f;
    if (target >= (int64_t)a.vocab && a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
    float factor = 0.0f, loss = 0.0f;
    if (target >= 0 && target < (int64_t)a.vocab && weight != 0.0f) {
      float most = -CUDART_INF_F;
      double others = 0.0;
      for (uint32_t i = 0; i < 8; ++i) most = fmaxf(most, part[i][lane].x), others += (double)part[i][lane].y;
      const float o = (float)others;
      const float raised = a.second ? a.raised[row] : 0.0f, right = exp2f(-raised), total = right + o;
      loss = weight * (raised == 0.0f ? log1pf(o) : logf(total) + raised * kLn2);
      factor = weight / total;
      a.kept[row * a.ldg + target] = __float2bfloat16_rn(-o);
      if (!a.second) {
        const bool wild = most > kWild && most < CUDART_INF_F;
        a.raised[row] = wild ? most : 0.0f;
        if (wild) {
          a.at_target[row] += most;
          a.wild[row / kWildRows] = 1;
          a.header->wild = 1;
        }
      }
    }
    a.loss[row] = late ? CUDART_NAN_F : loss;
    factors[lane] = factor;
  }
  __syncthreads();
  if (row0 + warp >= a.rows) return;
  const float f = factors[warp];
  if ((threadIdx.x & 31) == 0) a.factor[row0 + warp] = f;
  __nv_bfloat16* const to = a.scaled + (row0 + warp) * a.scaled_ld;
  auto scale = [&](uint32_t i, const uint4& raw) {
    float x[8] = {};
    if (f != 0.0f) {  // else the row may hold anything
      if (i + 8 <= a.dim) {
        widen<__nv_bfloat16>(raw, x);
      } else {
        for (uint32_t k = 0; i + k < a.dim; ++k) x[k] = to_float(h[i + k]);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= f;
    }
    *reinterpret_cast<uint4*>(to + i) = narrow<__nv_bfloat16>(x);
  };
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (at + k * 256 < a.dim) scale(at + k * 256, ahead[k]);
  for (uint32_t i = at + 1024; i < a.dim; i += 1024) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * 256 + 8 <= a.dim) ahead[k] = __ldg(reinterpret_cast<const uint4*>(h + i + k * 256));
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * 256 < a.dim) scale(i + k * 256, ahead[k]);
  }
}

// Few logits: they are there themselves, in parts of their sums, and a row's loss and G are made at once by THREADS threads, of which each holds up to 32 of them.
struct SoftmaxArgs {
  const float* parts;
  uint64_t split_stride, ldz, rows, ldg, hidden_ld, scaled_ld;
  uint32_t splits, vocab, token_bytes, dim;
  const void* targets;
  const float* weight;
  const float* up;  // multiplies the weight, or nullptr: up_by does
  float up_by, k2;
  float* loss;
  void* to;  // G; or nullptr: the loss alone
  const uint16_t* hidden;
  uint16_t* scaled;
  const Header* header;
  int32_t* status;
};
constexpr uint32_t kHeld = 8;  // times four logits of a thread
constexpr uint32_t kMostHeld = 256 * 4 * kHeld;
template <int THREADS, bool MAX>
__device__ __forceinline__ float over_row(float x, float* shared) {
#pragma unroll
  for (int d = 16; d; d /= 2) {
    const float y = __shfl_xor_sync(kFull, x, d);
    x = MAX ? fmaxf(x, y) : x + y;
  }
  if constexpr (THREADS > 32) {
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
    __syncthreads();
    x = shared[threadIdx.x % (THREADS / 32)];
#pragma unroll
    for (int d = THREADS / 64; d; d /= 2) {
      const float y = __shfl_xor_sync(kFull, x, d);
      x = MAX ? fmaxf(x, y) : x + y;
    }
  }
  return x;
}
template <class T, int THREADS>
__global__ void __launch_bounds__(256, 3) k_head_softmax(const SoftmaxArgs a) {
  pdl_enter();
  if (a.to) let_next_in();  // else the last of the call
  __shared__ float shared[2][8], at_target;
  const uint64_t row = THREADS == 32 ? (uint64_t)blockIdx.x * 8 + threadIdx.x / 32 : blockIdx.x;
  const uint32_t mine = threadIdx.x % THREADS;
  if (row >= a.rows) return;
  const int64_t word = target_of(a.targets, a.token_bytes, row);
  const float weight = a.weight ? a.weight[row] : 1.0f;
  uint32_t late = 0;
  for (uint32_t i = threadIdx.x & 31; i < kNumSM; i += 32) late |= a.header->late[i];
  constexpr uint32_t kAhead = THREADS == 32 ? 4 : 2;
  uint4 ahead[kAhead];  // the beginning of the hidden states, on its way meanwhile
  const uint16_t* const h = a.hidden + row * a.hidden_ld;
  if (a.to) {
#pragma unroll
    for (uint32_t k = 0; k < kAhead; ++k)
      if ((k * THREADS + mine) * 8 + 8 <= a.dim) ahead[k] = __ldg(reinterpret_cast<const uint4*>(h + (k * THREADS + mine) * 8));
  }
  float z[kHeld][4] = {};
  const float* const from = a.parts + row * a.ldz + mine * 4;
  auto part = [&](uint32_t i, uint32_t k) {
    return (i * THREADS + mine) * 4 < a.vocab && k < a.splits ? *reinterpret_cast<const float4*>(from + k * a.split_stride + i * THREADS * 4) : make_float4(0, 0, 0, 0);
  };
  auto add = [&](uint32_t i, const float4& x) { z[i][0] += x.x, z[i][1] += x.y, z[i][2] += x.z, z[i][3] += x.w; };
  if (a.splits >= 4) {  // many parts of few logits, or few of many: four or eight loads on their way
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i) {
      if (i * THREADS * 4 >= a.vocab) break;
      for (uint32_t k = 0; k < a.splits; k += 4) {
        const float4 x0 = part(i, k), x1 = part(i, k + 1), x2 = part(i, k + 2), x3 = part(i, k + 3);
        add(i, x0), add(i, x1), add(i, x2), add(i, x3);
      }
    }
  } else {
    for (uint32_t k = 0; k < a.splits; ++k)
#pragma unroll
      for (uint32_t i = 0; i < kHeld; ++i) {
        if (i * THREADS * 4 >= a.vocab) break;
        if ((i * THREADS + mine) * 4 < a.vocab) add(i, *reinterpret_cast<const float4*>(from + k * a.split_stride + i * THREADS * 4));
      }
  }
  if (word >= (int64_t)a.vocab && a.status && mine == 0) set_status(a.status, CVLC_ERR_INVALID_ARG);
  const bool there = word >= 0 && word < (int64_t)a.vocab && weight != 0.0f;
  const uint32_t target = there ? (uint32_t)word : 0;
  float most = -CUDART_INF_F, zt = 0.0f, o = 0.0f;
#pragma unroll
  for (uint32_t i = 0; i < kHeld; ++i) {
    if (i * THREADS * 4 >= a.vocab) break;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      const uint32_t col = (i * THREADS + mine) * 4 + k;
      z[i][k] = col < a.vocab ? z[i][k] * a.k2 : -CUDART_INF_F;
      most = fmaxf(most, z[i][k]);
      if (col == target) zt = z[i][k], z[i][k] = -CUDART_INF_F;
    }
  }
  if (THREADS > 32 && target / 4 % THREADS == mine) at_target = zt;
  most = over_row<THREADS, true>(most, shared[0]);
  zt = known(THREADS > 32 ? at_target : __shfl_sync(kFull, zt, target / 4 % 32));
#pragma unroll
  for (uint32_t i = 0; i < kHeld; ++i) {
    if (i * THREADS * 4 >= a.vocab) break;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      z[i][k] = exp2_fast(z[i][k] - most);
      o += z[i][k];
    }
  }
  o = over_row<THREADS, false>(o, shared[1]);
  const bool gone = __any_sync(kFull, late);
  const float right = exp2f(zt - most), total = right + o, w = gone ? CUDART_NAN_F : weight * (a.up ? *a.up : a.up_by);
  const float f = w / total, of_target = -(o / total) * w;
  if (mine == 0) a.loss[row] = gone ? CUDART_NAN_F : !there ? 0.0f : weight * (most == zt ? log1pf(o) : logf(total) + (most - zt) * kLn2);
  if (!a.to) return;
  T* const to = static_cast<T*>(a.to) + row * a.ldg + mine * 4;
#pragma unroll
  for (uint32_t i = 0; i < kHeld; ++i) {
    if (i * THREADS * 4 >= a.vocab) break;
    const uint32_t col = (i * THREADS + mine) * 4;
    float g[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) g[k] = !there ? 0.0f : col + k == target ? of_target : z[i][k] * f;
    if (col < a.vocab) *reinterpret_cast<uint2*>(to + i * THREADS * 4) = make_uint2(pack2<T>(g[0], g[1]), pack2<T>(g[2], g[3]));
  }
  uint16_t* const scaled = a.scaled + row * a.scaled_ld;
  uint32_t col = mine * 8;
#pragma unroll
  for (uint32_t k = 0; k < kAhead; ++k)
    if (col + 8 <= a.dim) {
      *reinterpret_cast<uint4*>(scaled + col) = there ? ahead[k] : make_uint4(0, 0, 0, 0);
      col += THREADS * 8;
    }
  masked_row(h, scaled, a.dim, there, col, THREADS);
}

// Exponentials that are kept relative to the maximum of their 128 columns become G: times exp(maximum - ln sum exp) and the weight.  In fp16 in their place; in fp32
// (up to 128 rows, where their room is small) so that G is rounded once.  A warp a row, two times 128 columns at a time.
struct RescaleArgs {
  const void* kept;
  void* to;
  uint64_t ld_kept, ld_to, rows, stats_stride;
  const float2* stats;
  const float4* row;
  const void* targets;
  uint32_t vocab, tile_n, token_bytes;
};
template <class FROM, class T>
__global__ void __launch_bounds__(256) k_head_rescale(const RescaleArgs a) {
  pdl_enter();
  let_next_in();
  const uint64_t row = (uint64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const uint32_t lane = threadIdx.x & 31;
  if (row >= a.rows) return;
  const float4 r = a.row[row];
  const FROM* const from = static_cast<const FROM*>(a.kept) + row * a.ld_kept;
  T* const to = static_cast<T*>(a.to) + row * a.ld_to;
  const int64_t target = r.y == 0.0f ? -1 : target_of(a.targets, a.token_bytes, row);
#pragma unroll 4
  for (uint32_t col = (blockIdx.y * 32 + lane) * 8; col < a.vocab; col += gridDim.y * 256) {
    const uint32_t tile = col / a.tile_n, slot = 2 * tile + (col - tile * a.tile_n) / 128;
    float v[8];
    if constexpr (std::is_same<FROM, float>::value) {
      const uint4 x = *reinterpret_cast<const uint4*>(from + col), y = *reinterpret_cast<const uint4*>(from + col + 4);
      float lo[4], hi[4];
      widen<float>(x, lo), widen<float>(y, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = lo[i], v[4 + i] = hi[i];
    } else {
      widen<FROM>(__ldcs(reinterpret_cast<const uint4*>(from + col)), v);
    }
    const float f = exp2f(a.stats[slot * a.stats_stride + row].x - r.x) * r.y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = r.y == 0.0f ? 0.0f : v[i] * f;
      if (target == (int64_t)col + i) v[i] = r.z;
    }
    *reinterpret_cast<uint4*>(to + col) = narrow<T>(v);
  }
}

struct JoinJob {
  const float* parts;
  uint64_t split_stride, ldp, ldo;
  uint32_t splits, dim;
  uint64_t rows;
  float alpha;
  const float *factor, *down;  // of a row; of all; or nullptr
  void* out;
};
struct JoinArgs {
  JoinJob of[2];
  uint32_t blocks;  // of the first
  const Header* header;
};
// The parts of the hidden states' gradient, and of the head's where it comes in parts, added up in their order, four columns a thread; with many parts (few rows) eight threads share them.
template <class T, int SHARE>
__global__ void __launch_bounds__(256) k_head_join(const __grid_constant__ JoinArgs all) {
  pdl_enter();
  __shared__ float4 share[SHARE > 1 ? 256 : 1];
  const bool late = any_late(all.header);
  const bool second = blockIdx.x >= all.blocks;
  const JoinJob& a = all.of[second];
  const uint32_t per = (a.dim + 3) / 4, of = 256 / SHARE, mine = threadIdx.x / of;
  const uint64_t i = (uint64_t)(blockIdx.x - (second ? all.blocks : 0)) * of + threadIdx.x % of, row = i / per;
  const uint32_t col = (uint32_t)(i - row * per) * 4;
  float4 s = make_float4(0, 0, 0, 0);
  if (row < a.rows) {
    const float* const from = a.parts + row * a.ldp + col;
#pragma unroll 8
    for (uint32_t k = mine; k < a.splits; k += SHARE) {
      const float4 x = *reinterpret_cast<const float4*>(from + k * a.split_stride);
      s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
  }
  if (SHARE > 1) {
    share[threadIdx.x] = s;
    __syncthreads();
    if (mine) return;
    for (uint32_t k = 1; k < SHARE; ++k) {
      const float4 x = share[k * of + threadIdx.x];
      s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
  }
  if (row >= a.rows) return;
  const float alpha = late ? CUDART_NAN_F : a.alpha * (a.factor ? a.factor[row] : a.down ? *a.down : 1.0f);
  T* const out = static_cast<T*>(a.out) + row * a.ldo + col;
  const float v[4] = {s.x * alpha, s.y * alpha, s.z * alpha, s.w * alpha};
  if (col + 4 <= a.dim && (reinterpret_cast<uintptr_t>(out) & 7) == 0) {
    *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (col + k < a.dim) out[k] = from_float<T>(v[k]);
  }
}

// ---- layout and launching --------------------------------------------------------------------

bool on16(const void* p, uint64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; }
uint32_t tiles(uint64_t n, uint32_t tile) { return (uint32_t)((n + tile - 1) / tile); }
// Up to 128 rows a block has them all; above, a pair of blocks reads half as much of the other operand.
bool by_pairs(uint64_t m) { return m > kTileM; }

// Rows that fit in one tile: the head is read once, by the SMs alike if its tiles come out even.
uint32_t stats_tile(uint64_t m, uint32_t n) {
  uint32_t best = kTileN;
  if (by_pairs(m)) return best;
  auto cost = [&](uint32_t t) { return (uint64_t)tiles(tiles(n, t), kNumSM) * t; };
  for (uint32_t t = kTileN; t >= 128; t -= 32)
    if (cost(t) < cost(best)) best = t;
  return best;
}
// In how many parts a sum is cut: as many as leave the SMs the least to do one behind the other.  A step of 64 takes 0.3 us, a part more costs its
// writing and reading.
uint32_t splits_of(uint64_t m, uint64_t n, uint32_t k_blocks, bool pairs) {
  const uint64_t all = (uint64_t)tiles(m, pairs ? 2 * kTileM : kTileM) * tiles(n, kTileN), at_once = pairs ? kNumSM / 2 : kNumSM;
  const double more = (double)(m * n) * 8 / 6.4e6 / 0.3 + 0.1;
  uint32_t best = 1;
  double cost = 1e30;
  for (uint32_t s = 1; s <= 64 && s * 8 <= (k_blocks > 8 ? k_blocks : 8); ++s) {
    const double c = (double)((all * s + at_once - 1) / at_once) / s * k_blocks + more * s;
    if (c < cost * 0.99) cost = c, best = s;
  }
  return best;
}

// Few logits, of which single blocks make tiles of any width: both at once.  A step takes 0.08 us and what it copies, a tile its reading and writing.
void cut_few(uint64_t m, uint64_t n, uint32_t k_blocks, uint32_t* tile_n, uint32_t* splits) {
  double cost = 1e30;
  for (uint32_t t = kTileN; t >= 32; t -= 32)
    for (uint32_t s = 1; s <= 32 && s <= k_blocks; ++s) {
      const uint64_t waves = ((uint64_t)tiles(m, kTileM) * tiles(n, t) * s + kNumSM - 1) / kNumSM;
      const double step = 0.08 + 0.0006 * ((m < kTileM ? m : kTileM) + t);
      const double c = (double)waves * (((k_blocks + s - 1) / s) * step + 0.5 + 0.004 * t) + s * (0.05 + (double)(m * n) * 8 / 6.4e6);
      if (c < cost * 0.99) cost = c, *tile_n = t, *splits = s;
    }
}

// What becomes of the exponentials of the first product.  Several pieces: nothing, there is no room for them.  Up to 128 rows: kept in fp32.  bf16 has fp32's
// range, and they are relative to the target's; fp16 has not, and they are relative to the maximum of 128 columns and gone over once more (777 x 1000 x
// 50021: 27 us; multiplying again 103).
constexpr uint64_t kLeastPiece = 1ull << 22;
// Few logits go through the memory in 32 bits: nothing has to be known of a row before its logits are there, none gets a second turn, and sums are cut
// wherever SMs are idle.  A step takes four launches instead of five (up to 128 rows) or eight: 149 x 624 x 56 39 -> 20 us, 5579 x 104 x 117 69 -> 25, 1518 x 1328 x
// 3047 even; a loss two as before: 3420 x 3856 x 101 30 -> 15, even at a million logits, 2252 x 94 x 3405 21 -> 29.
constexpr uint64_t kFewLogits = kLeastPiece, kFewOfLoss = 1ull << 20;
enum class Keep { kNot, kFew, kWide, kBf16, kFp16 };
struct HeadLayout {
  Keep keep;
  bool pairs;              // in the gradients' products
  bool whole;              // d_hidden is made in one part and needs no joining
  bool copy_hidden, copy_head;
  uint64_t ld;             // of copies
  uint32_t piece, pieces;  // words
  uint64_t ldg, ldp, stats_stride;
  uint32_t splits, slots, blocks_wild;
  uint64_t ldz;  // few logits
  uint32_t tile_z, splits_z, splits_head;
  size_t off_z, off_head_parts, off_hidden, off_head, off_scaled, off_stats, off_target, off_row, off_factor, off_raised, off_wild, off_g, off_wide, off_parts, total;
};
HeadLayout head_layout(const cvlc_head& a, uint32_t pieces) {
  HeadLayout L = {};
  if (pieces) {
    // a piece of less than 4 M logits is not worth its launches (22 x 1533 x 2387 in five pieces 119 us, in one 46)
    const uint64_t words = ((uint64_t)a.vocab + pieces - 1) / pieces, least = a.rows ? (kLeastPiece + a.rows - 1) / a.rows : 1;
    L.piece = tiles(words > least ? words : least < a.vocab ? least : a.vocab, kTileN) * kTileN;
    L.pieces = tiles(a.vocab, L.piece);
    if (L.pieces == 1) L.piece = a.vocab;
  }
  const bool few = L.pieces <= 1 && a.vocab <= kMostHeld && a.rows * a.vocab <= (pieces ? kFewLogits : kFewOfLoss);
  L.keep = few ? Keep::kFew : L.pieces != 1 ? Keep::kNot : !by_pairs(a.rows) ? Keep::kWide : a.dtype == CVLC_BF16 ? Keep::kBf16 : Keep::kFp16;
  L.pairs = !few && by_pairs(a.rows);
  // copied where they do not begin on 16 bytes, or where rows that count for nothing have to become zeros first
  L.copy_hidden = !on16(a.hidden_dev, a.hidden_stride) || (pieces && (L.keep == Keep::kNot || L.keep == Keep::kFp16));
  L.copy_head = !on16(a.head_dev, a.head_stride);
  L.ld = (a.dim + 7) / 8 * 8;
  L.stats_stride = (a.rows + 31) / 32 * 32;
  size_t at = align256(sizeof(Header));
  auto take = [&](size_t bytes) { const size_t from = at; at = align256(at + bytes); return from; };
  L.off_hidden = take(L.copy_hidden ? a.rows * L.ld * 2 : 0);
  L.off_head = take(L.copy_head ? a.vocab * L.ld * 2 : 0);
  if (few) {
    L.ldz = (uint64_t)tiles(a.vocab, 32) * 32;
    cut_few(a.rows, a.vocab, tiles(a.dim, kTileK), &L.tile_z, &L.splits_z);
    L.off_z = take((size_t)L.splits_z * a.rows * L.ldz * 4);
  } else {
    L.slots = 2 * tiles(a.vocab, stats_tile(a.rows, a.vocab));
    L.off_stats = take((size_t)L.slots * L.stats_stride * 8);
    L.off_target = take(a.rows * 4);
  }
  if (pieces) {
    L.ldg = (uint64_t)tiles(L.piece, 32) * 32;
    L.ldp = (a.dim + 31) / 32 * 32;
    L.splits = splits_of(a.rows, a.dim, tiles(L.piece, kTileK), L.pairs);
    // of few words and many rows the head's gradient has few tiles and long sums (7094 x 144 x 83: 79 -> 34 us)
    L.splits_head = few ? splits_of(a.vocab, a.dim, tiles(a.rows, kTileK), false) : 1;
    L.whole = few && L.splits == 1;
    if (L.splits_head > 1) L.off_head_parts = take((size_t)L.splits_head * a.vocab * L.ldp * 4);
    L.off_g = take(a.rows * L.ldg * 2);
    if (!L.whole) L.off_parts = take((size_t)L.splits * a.rows * L.ldp * 4);
    if (L.keep == Keep::kBf16) {
      L.blocks_wild = tiles(a.rows, kWildRows);
      L.off_scaled = take(a.rows * L.ld * 2);
      L.off_factor = take(a.rows * 4);
      L.off_raised = take(a.rows * 4);
      L.off_wild = take(L.blocks_wild * 4);
    } else if (!few) {
      L.off_row = take(a.rows * 16);
    }
    if (few || L.keep == Keep::kWide) L.off_scaled = take(a.rows * L.ld * 2);
    if (L.keep == Keep::kWide) L.off_wide = take(a.rows * L.ldg * 4);
  }
  L.total = at;
  return L;
}

template <int EPI, bool A_ROWS, bool B_ROWS, class T, int CG>
cudaError_t run_product_of(int id, const Products<EPI>& g, uint64_t items, cudaStream_t st, bool overlap) {
  static OncePerDevice once;
  const cudaError_t e = once_per_device(once, [] { return allow_shared(k_head_product<EPI, A_ROWS, B_ROWS, T, CG>, kGemmShared); });
  if (e != cudaSuccess) return e;
  LaunchScope ls(id, st);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)(items * CG < kNumSM ? items * CG : kNumSM));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kGemmShared;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = overlap ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, k_head_product<EPI, A_ROWS, B_ROWS, T, CG>, Products<EPI>(g));
  return cudaGetLastError();
}
struct Operand {
  const void* at;
  uint64_t cols, rows, ld;
};
void set_stages(Product& g, uint32_t stage_bytes) {
  g.stage_bytes = stage_bytes;
  g.stages = kRingBytes / stage_bytes < kMostStages ? kRingBytes / stage_bytes : kMostStages;
}
// D = A B^T, sums along the operands' columns, or along their rows
bool make_product(Product& g, bool bf16, bool pairs, const Operand& a, bool a_rows, const Operand& b, bool b_rows, bool boxes) {
  if (!g.tile_n) g.tile_n = kTileN;
  g.tiles_m = tiles(g.m, pairs ? 2 * kTileM : kTileM), g.tiles_n = tiles(g.n, g.tile_n);
  // Of the operand with fewer tiles a group, 32 MB or eight tiles, stays in the L2 cache (of which each half of the chip has its own copy), while the other
  // one's pass by.  (All of it at once, 67 MB: 8192 x 4096 x 16384 read 1.2 GB of memory instead of 0.43 for the logits.)
  g.m_first = g.tiles_m <= g.tiles_n;
  const uint64_t bytes = (uint64_t)2 * kTileN * kTileK * ((g.k_blocks + g.splits - 1) / g.splits);
  g.group = (uint32_t)((32ull << 20) / bytes);
  if (g.group < 8) g.group = 8;
  const uint32_t fewer = g.m_first ? g.tiles_m : g.tiles_n;
  if (g.group > fewer) g.group = fewer;
  // what a block copies at a time: of the rows those that are there, of the sum (rows first) what there is
  const uint32_t rows = !pairs && !a_rows && g.m < kTileM ? (g.m + 7) / 8 * 8 : kTileM, columns = g.tile_n / (pairs ? 2 : 1);
  g.values = !pairs && a_rows && b_rows && a.rows < kTileK ? (uint32_t)(a.rows + 15) / 16 * 16 : kTileK;
  g.a_bytes = rows * g.values * 2, g.b_bytes = columns * g.values * 2, g.stage_bytes = g.a_bytes + g.b_bytes;
  set_stages(g, g.stage_bytes);
  if (boxes && !make_tensor_map(&g.c, g.out, bf16, g.n, g.m, g.ldo, 64, 32)) return false;
  return make_tensor_map(&g.a, a.at, bf16, a.cols, a.rows, a.ld, 64, a_rows ? g.values : rows) &&
         make_tensor_map(&g.b, b.at, bf16, b.cols, b.rows, b.ld, 64, b_rows ? g.values : columns);
}

struct Gradients {
  void* d_hidden;
  uint64_t d_hidden_stride;
  void* d_head;
  uint64_t d_head_stride;
};

template <class T>
struct HeadRun {
  const cvlc_head& a;
  const HeadLayout L;
  uint8_t* const base;
  const cudaStream_t st;
  Header* const header;
  Operand hidden, head;
  const HeadFault* const fault;
  bool behind = false;  // some kernel of the call is in front
  uint32_t products = 0;  // launched so far
  cudaError_t error = cudaSuccess;

  HeadRun(const cvlc_head& a_, uint32_t pieces, void* ws, cudaStream_t st_, const HeadFault* fault_)
      : a(a_), L(head_layout(a_, pieces)), base(static_cast<uint8_t*>(ws)), st(st_), header(static_cast<Header*>(ws)),
        hidden{a_.hidden_dev, a_.dim, a_.rows, a_.hidden_stride}, head{a_.head_dev, a_.dim, a_.vocab, a_.head_stride}, fault(fault_) {}
  template <class P>
  P* at(size_t off) const { return reinterpret_cast<P*>(base + off); }
  template <class... Params, class... Args>
  void launch(int id, void (*kernel)(Params...), uint32_t grid, uint32_t threads, Args&&... args) {
    launch_kernel(id, kernel, dim3(grid), dim3(threads), 0, st, behind, args...);
    behind = true;
  }
  // What a product's logit is multiplied by.  The tensor cores cut off at each step of 16 of a sum, on average half a unit of fp32's last place of the sum so far; of sums
  // that grow evenly that makes a quarter of 2^-24 a step, which is put back (losses at dim 4096 were 2.2e-6 off without, 0.8e-6 with it; the worst, all of a sum in
  // its first value or in its last, 6.6e-6 and 0.1e-6 without, 2.8e-6 and 3.7e-6).
  float logit_scale() const {
    const double steps = (a.dim + 15) / 16 / (double)(L.keep == Keep::kFew ? L.splits_z : 1);
    return (float)((double)a.scale * 1.4426950408889634 * (1.0 + steps * 0.25 * 0x1p-24));
  }
  Product product() const {
    Product p = {};
    p.splits = 1, p.alpha = a.scale, p.k2 = logit_scale(), p.targets = a.targets_dev, p.token_bytes = a.token_bytes;
    p.stats = at<float2>(L.off_stats), p.stats_stride = L.stats_stride, p.at_target = at<float>(L.off_target);
    p.header = header, p.status = a.status_dev, p.lost_copy = p.lost_tile = ~0u, p.most = kMostWait;
    return p;
  }
  static constexpr bool bf16 = std::is_same<T, __nv_bfloat16>::value;
  template <int EPI, bool A_ROWS, bool B_ROWS, int CG>
  void run_product(int id, Products<EPI> p, bool fits) {
    if (fault && products == fault->product) p.p[0].lost_copy = fault->copy, p.p[0].lost_tile = fault->tile, p.p[0].most = fault->most;
    ++products;
    uint64_t items = 0;
    for (const Product& x : p.p) items += (uint64_t)x.tiles_m * x.tiles_n * x.splits;
    if (error == cudaSuccess) error = fits ? run_product_of<EPI, A_ROWS, B_ROWS, T, CG>(id, p, items, st, behind) : cudaErrorUnknown;
    behind = true;
  }
  // a product of hidden rows with words
  template <int EPI>
  void multiply(int id, Product p, const Operand& words) {
    const bool pairs = by_pairs(a.rows), fits = make_product(p, bf16, pairs, hidden, false, words, false, EPI != kStats && EPI != kKeepWide);
    if constexpr (EPI != kKeepWide)
      if (pairs) run_product<EPI, false, false, 2>(id, {{p}}, fits);
    if constexpr (EPI != kKeep && EPI != kKeepOwn)
      if (!pairs) run_product<EPI, false, false, 1>(id, {{p}}, fits);
  }
  // the copies of rows that do not lie on 16 bytes, or (targets) of those that may not count
  void copies(const void* targets) {
    AlignArgs r = {};
    uint32_t n = 0, blocks = 0;
    auto add = [&](Operand& x, size_t off, const void* t) {
      r.of[n++] = {static_cast<const uint16_t*>(x.at), at<uint16_t>(off), x.ld, L.ld, x.rows, t};
      if (n == 1) r.blocks = tiles(x.rows, 8);
      blocks += tiles(x.rows, 8);
      x.at = base + off, x.ld = L.ld;
    };
    if (L.copy_hidden) add(hidden, L.off_hidden, targets);
    if (L.copy_head) add(head, L.off_head, nullptr);
    r.dim = a.dim, r.token_bytes = a.token_bytes, r.vocab = a.vocab, r.weight = a.row_weight_dev;
    if (n) launch(kKHeadAlign, k_head_align, blocks, 256, r);
  }
  RowsArgs rows(float* loss) const {
    RowsArgs r = {};
    r.stats = at<float2>(L.off_stats), r.stats_stride = L.stats_stride, r.slots = L.slots, r.token_bytes = a.token_bytes, r.vocab = a.vocab;
    r.at_target = at<float>(L.off_target), r.targets = a.targets_dev, r.weight = a.row_weight_dev, r.loss = loss, r.header = header, r.rows = a.rows;
    r.status = a.status_dev;
    return r;
  }
  uint32_t row_blocks() const { return tiles(a.rows, kRowsOf); }

  // the losses, and what makes G of the logits
  void logits_once(float* loss, bool graded) {
    Product p = product();
    p.m = (uint32_t)a.rows, p.n = a.vocab, p.k_blocks = tiles(a.dim, kTileK), p.first = 1, p.tile_n = stats_tile(a.rows, a.vocab);
    p.out = base + (L.keep == Keep::kWide ? L.off_wide : L.off_g), p.ldo = L.ldg;
    if (graded && L.keep == Keep::kWide) multiply<kKeepWide>(kKHeadKeep, p, head);
    else if (!graded || L.keep == Keep::kNot) multiply<kStats>(kKHeadStats, p, head);
    else if constexpr (!bf16) multiply<kKeepOwn>(kKHeadKeep, p, head);
    RowsArgs r = rows(loss);
    r.row = graded ? at<float4>(L.off_row) : nullptr, r.up = graded ? up() : nullptr, r.up_by = up_by();
    if (graded && L.keep == Keep::kWide)
      r.hidden = static_cast<const __nv_bfloat16*>(hidden.at), r.hidden_ld = hidden.ld, r.scaled = at<__nv_bfloat16>(L.off_scaled), r.scaled_ld = L.ld, r.dim = a.dim;
    launch(kKHeadRows, k_head_rows, row_blocks(), 256, r);
  }
  template <class FROM>
  void rescale(size_t from) {
    RescaleArgs r = {};
    r.kept = base + from, r.to = base + L.off_g, r.ld_kept = r.ld_to = L.ldg, r.rows = a.rows, r.stats_stride = L.stats_stride, r.stats = at<float2>(L.off_stats);
    r.row = at<float4>(L.off_row), r.targets = a.targets_dev, r.vocab = a.vocab, r.tile_n = stats_tile(a.rows, a.vocab), r.token_bytes = a.token_bytes;
    const uint32_t blocks = tiles(a.rows, 8), along = tiles(a.vocab, 256), most = blocks < 8 * kNumSM ? tiles(8 * kNumSM, blocks) : 1;
    if (error == cudaSuccess)
      launch_kernel(kKHeadRescale, k_head_rescale<FROM, T>, dim3(blocks, along < most ? along : most), dim3(256), 0, st, true, r);
  }
  // The part of a piece of the words in both gradients.  Up to 128 rows, where the hidden states' gradient has few tiles and the head's tiles are one step
  // of the sum each, one launch makes both (16 x 1024 x 32000: 52 -> 30 us); by pairs, two do (8192 x 4096 x 131072: 13.7 ms, 15.2 in one).
  void gradients(uint32_t from, uint32_t words, const Operand& hidden_scaled, const Gradients& to) {
    const Operand g = {base + L.off_g, words, a.rows, L.ldg}, piece = {static_cast<const T*>(head.at) + (uint64_t)from * head.ld, a.dim, words, head.ld};
    const bool pairs = L.pairs;
    Product p = product();
    p.m = (uint32_t)a.rows, p.n = a.dim, p.k_blocks = tiles(words, kTileK);
    p.splits = L.splits <= p.k_blocks ? L.splits : p.k_blocks;
    p.out = base + L.off_parts, p.ldo = L.ldp, p.split_stride = a.rows * L.ldp, p.add = from != 0;
    Product q = product();
    q.m = words, q.n = a.dim, q.k_blocks = tiles(a.rows, kTileK), q.splits = L.splits_head;
    T* const out = static_cast<T*>(to.d_head) + (uint64_t)from * to.d_head_stride;
    q.out = out, q.ldo = to.d_head_stride, q.wide = on16(out, to.d_head_stride) && a.dim % 8 == 0;  // a box writes whole vectors of 16 bytes: what lies behind a row's end with them, too
    q.alpha = a.scale * down_by(), q.alpha_dev = down();
    q.whole = q.splits == 1;
    if (L.whole)
      p.whole = 1, p.out = to.d_hidden, p.ldo = to.d_hidden_stride, p.wide = on16(to.d_hidden, to.d_hidden_stride) && a.dim % 8 == 0, p.alpha = q.alpha, p.alpha_dev = q.alpha_dev;
    if (q.splits > 1) q.out = base + L.off_head_parts, q.ldo = L.ldp, q.split_stride = words * L.ldp, q.wide = 0;
    const bool fits = make_product(p, bf16, pairs, g, false, piece, true, p.wide) && make_product(q, bf16, pairs, g, true, hidden_scaled, true, q.wide);
    if (pairs) {
      run_product<kParts, false, true, 2>(kKHeadParts, {{p}}, fits);
      run_product<kGrad, true, true, 2>(kKHeadGrad, {{q}}, fits);
    } else {
      set_stages(p, p.stage_bytes > q.stage_bytes ? p.stage_bytes : q.stage_bytes);  // one ring for both
      run_product<kBoth, false, true, 1>(kKHeadGrads, {{p, q}}, fits);
    }
  }
  void join(const Gradients& to, const float* factor) {
    JoinArgs j = {};
    uint64_t quads[2] = {};
    uint32_t n = 0;
    auto add = [&](size_t parts, uint32_t splits, uint64_t rows, void* out, uint64_t stride) {
      JoinJob& x = j.of[n];
      x.parts = at<float>(parts), x.split_stride = rows * L.ldp, x.ldp = L.ldp, x.ldo = stride, x.splits = splits, x.dim = a.dim, x.rows = rows, x.alpha = a.scale * down_by();
      x.factor = factor, x.down = down(), x.out = out, quads[n++] = rows * ((a.dim + 3) / 4);
    };
    if (!L.whole) add(L.off_parts, L.splits, a.rows, to.d_hidden, to.d_hidden_stride);
    if (L.splits_head > 1) add(L.off_head_parts, L.splits_head, a.vocab, to.d_head, to.d_head_stride);
    if (!n) return;
    j.header = header;
    const bool shared = (L.splits >= 8 || L.splits_head >= 8) && quads[0] + quads[1] <= 32768;
    const uint32_t of = shared ? 32 : 256;
    j.blocks = (uint32_t)((quads[0] + of - 1) / of);
    const uint32_t blocks = j.blocks + (uint32_t)((quads[1] + of - 1) / of);
    if (shared) launch(kKHeadJoin, k_head_join<T, 8>, blocks, 256, j);
    else launch(kKHeadJoin, k_head_join<T, 1>, blocks, 256, j);
  }
  // fp16: by how much G is raised, known beforehand where no row has a weight
  bool weighed() const { return !bf16 && a.row_weight_dev; }
  const float* up() const { return weighed() ? &header->up : nullptr; }
  const float* down() const { return weighed() ? &header->down : nullptr; }
  static constexpr float up_by() { return bf16 ? 1.0f : 0x1p15f; }
  float down_by() const { return bf16 || weighed() ? 1.0f : 0x1p-15f; }
  void begin() {
    if (weighed()) launch(kKHeadBegin, k_head_begin, 1, a.rows > 256 ? 1024 : 256, header, a.row_weight_dev, a.targets_dev, a.token_bytes, a.rows, a.vocab);
  }
  void run_few(float* loss, const Gradients* to) {
    if (to) begin();
    Product p = product();
    p.m = (uint32_t)a.rows, p.n = a.vocab, p.k_blocks = tiles(a.dim, kTileK), p.first = 1, p.tile_n = L.tile_z, p.splits = L.splits_z;
    p.out = base + L.off_z, p.ldo = L.ldz, p.split_stride = a.rows * L.ldz;
    const bool fits = make_product(p, bf16, false, hidden, false, head, false, false);
    run_product<kParts, false, false, 1>(kKHeadLogits, {{p}}, fits);
    SoftmaxArgs r = {};
    r.parts = at<float>(L.off_z), r.split_stride = p.split_stride, r.ldz = L.ldz, r.rows = a.rows, r.ldg = L.ldg, r.hidden_ld = hidden.ld, r.scaled_ld = L.ld;
    r.splits = L.splits_z, r.vocab = a.vocab, r.token_bytes = a.token_bytes, r.dim = a.dim, r.targets = a.targets_dev, r.weight = a.row_weight_dev;
    r.up = to ? up() : nullptr, r.up_by = up_by(), r.k2 = p.k2, r.loss = loss, r.to = to ? base + L.off_g : nullptr;
    r.hidden = static_cast<const uint16_t*>(hidden.at), r.scaled = at<uint16_t>(L.off_scaled), r.header = header, r.status = a.status_dev;
    // as many threads a row as hold it, and more while there is work for them and all rows' are resident (50 x 768 x 1000: 29 us by 32, 20 by 256; 700 x 700 x 300: 28, 26 by 128, 29 by 256;
    // 7094 x 144 x 83: 25 by 32, 47 by 256)
    uint32_t threads = 32;
    const uint32_t work = to && a.dim / 2 > a.vocab ? a.dim / 2 : a.vocab;  // logits or, at 16 bytes a thread, hidden states
    while (threads < 256 && (a.vocab > threads * 4 * kHeld || (work > threads * 4 && a.rows * threads * 2 <= kNumSM * 1024))) threads *= 2;
    if (threads == 32) launch(kKHeadSoftmax, k_head_softmax<T, 32>, tiles(a.rows, 8), 256, r);
    else if (threads == 64) launch(kKHeadSoftmax, k_head_softmax<T, 64>, (uint32_t)a.rows, 64, r);
    else if (threads == 128) launch(kKHeadSoftmax, k_head_softmax<T, 128>, (uint32_t)a.rows, 128, r);
    else launch(kKHeadSoftmax, k_head_softmax<T, 256>, (uint32_t)a.rows, 256, r);
    if (!to) return;
    gradients(0, a.vocab, {base + L.off_scaled, a.dim, a.rows, L.ld}, *to);
    join(*to, nullptr);
  }
  void run_kept(float* loss, const Gradients& to) {
    TargetArgs t = {};
    t.hidden = hidden.at, t.head = head.at, t.targets = a.targets_dev, t.hidden_ld = hidden.ld, t.head_ld = head.ld, t.rows = a.rows, t.dim = a.dim;
    t.vocab = a.vocab, t.token_bytes = a.token_bytes, t.blocks_wild = L.blocks_wild, t.weight = a.row_weight_dev, t.at_target = at<float>(L.off_target);
    t.k2 = a.scale * kLog2E, t.wild = at<uint32_t>(L.off_wild), t.header = header;
    launch(kKHeadTarget, k_head_target, tiles(a.rows, 8), 256, t);
    for (uint32_t turn = 0; turn < 2; ++turn) {
      Product p = product();
      p.m = (uint32_t)a.rows, p.n = a.vocab, p.k_blocks = tiles(a.dim, kTileK), p.first = turn == 0;
      p.out = base + L.off_g, p.ldo = L.ldg;
      p.early = turn == 0;  // k_head_target, in front, writes none of the operands, and the copies of rows, if any, are complete: it has waited for them
      if (turn) p.skip = &header->wild, p.wild = t.wild;
      if constexpr (bf16) multiply<kKeep>(kKHeadKeep, p, head);
      RowsArgs r = rows(loss);
      r.kept = at<__nv_bfloat16>(L.off_g), r.ldg = L.ldg, r.hidden = static_cast<const __nv_bfloat16*>(hidden.at), r.hidden_ld = hidden.ld;
      r.scaled = at<__nv_bfloat16>(L.off_scaled), r.scaled_ld = L.ld, r.factor = at<float>(L.off_factor), r.raised = at<float>(L.off_raised), r.wild = t.wild;
      r.dim = a.dim, r.second = turn;
      launch(kKHeadRows, k_head_rows_kept, row_blocks(), 256, r);
    }
    gradients(0, a.vocab, {base + L.off_scaled, a.dim, a.rows, L.ld}, to);
    join(to, at<float>(L.off_factor));
  }
  void run_pieces(float* loss, const Gradients& to) {
    begin();
    copies(L.keep == Keep::kWide ? nullptr : a.targets_dev);
    logits_once(loss, true);
    if (L.keep == Keep::kWide) rescale<float>(L.off_wide);
    else if constexpr (!bf16)
      if (L.keep == Keep::kFp16) rescale<T>(L.off_g);
    const Operand counted = L.keep == Keep::kWide ? Operand{base + L.off_scaled, a.dim, a.rows, L.ld} : hidden;
    for (uint32_t i = 0; i < L.pieces; ++i) {
      const uint32_t from = i * L.piece, words = i + 1 < L.pieces ? L.piece : a.vocab - from;
      if (L.keep == Keep::kNot) {
        Product p = product();
        p.m = (uint32_t)a.rows, p.n = words, p.k_blocks = tiles(a.dim, kTileK), p.col0 = from, p.row = at<float4>(L.off_row);
        p.out = base + L.off_g, p.ldo = L.ldg;
        multiply<kProbs>(kKHeadProbs, p, {static_cast<const T*>(head.at) + (uint64_t)from * head.ld, a.dim, words, head.ld});
      }
      gradients(from, words, counted, to);
    }
    join(to, nullptr);
  }
  cudaError_t run(float* loss, const Gradients* to) {
    if (!to || L.keep == Keep::kBf16 || L.keep == Keep::kFew) copies(nullptr);
    if (L.keep == Keep::kFew) run_few(loss, to);
    else if (!to) logits_once(loss, false);
    else if (L.keep == Keep::kBf16) run_kept(loss, *to);
    else run_pieces(loss, *to);
    return error != cudaSuccess ? error : cudaGetLastError();
  }
};

}  // namespace

size_t head_ws_bytes(const cvlc_head& a, uint32_t pieces) { return head_layout(a, pieces).total; }

cudaError_t launch_head(const cvlc_head& a, uint32_t pieces, float* loss, void* d_hidden, uint64_t d_hidden_stride, void* d_head, uint64_t d_head_stride, void* ws,
                        cudaStream_t st, const HeadFault* fault) {
  const Gradients g = {d_hidden, d_hidden_stride, d_head, d_head_stride};
  if (a.dtype == CVLC_F16) return HeadRun<__half>(a, pieces, ws, st, fault).run(loss, pieces ? &g : nullptr);
  return HeadRun<__nv_bfloat16>(a, pieces, ws, st, fault).run(loss, pieces ? &g : nullptr);
}

}  // namespace cvlc
