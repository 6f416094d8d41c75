// Softmax cross entropy of hidden states against a head matrix, and its gradients, without the logits.
//
// z_tv = scale h_t . w_v;  loss_t = weight_t (ln sum_v exp(z_tv) - z_t,target);  G_tv = weight_t (q_tv - [v = target]);
// dh_t = scale sum_v G_tv w_v;  dw_v = scale sum_t G_tv h_t
//
// Three products of rows x vocab x dim each.  The first one's values never leave the tensor memory: a tile of them becomes, per row, its maximum
// and its sum of exponentials (k_head_stats), which are joined to the row's loss and ln sum exp (k_head_rows).  For the gradients a piece of the
// vocabulary at a time is multiplied again and becomes G, rounded to the type of the operands (k_head_probs), from which come the piece of the head's
// gradient (k_head_grad) and the piece's part of the hidden states' (k_head_parts, in fp32, joined by k_head_join).
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

// ---- the products --------------------------------------------------------------------------
// A block has a tile of 128 rows by 256 columns: one thread copies operands (a ring of stages of 64 values of the sum), one issues the
// products, eight warps read a finished tile from the tensor memory while the next one is made in its other half.
constexpr uint32_t kTileM = 128, kTileN = 256, kTileK = 64;
constexpr int kThreads = 384, kOutWarps = 8;
constexpr uint32_t kBytesA = kTileM * kTileK * 2, kBytesB = kTileN * kTileK * 2;
constexpr int kStages = 4;
constexpr size_t kGemmShared = kStages * (kBytesA + kBytesB) + 1024;

enum Epilogue { kStats, kProbs, kParts, kGrad };
struct Product {
  CUtensorMap a, b;
  uint32_t m, n, k_blocks;               // rows, columns, steps of 64 of the sum
  uint32_t tiles_m, tiles_n, splits;     // of the sum
  uint32_t m_first;                      // tiles of one column of tiles follow one another, else those of a row
  uint32_t col0, token_bytes;            // stats, probs: the word of column 0
  float k2, alpha;                       // scale log2(e); factor of the output
  const void* targets;
  float2* stats;                         // (maximum, sum relative to it) of a row's half tile
  float* at_target;                      // z of the row's target, in log2
  uint64_t stats_stride;
  const float4* row;                     // probs: what makes a row's G of its z
  void* out;
  uint64_t ldo, split_stride;
  uint32_t add, wide;                    // added to what is there; rows of `out` by vectors of 32 bytes
  const float* alpha_dev;                // or nullptr; multiplies alpha
  int32_t *late, *status;
};

struct Work {
  uint32_t m0, n0, k_from, k_to, split;
};
__device__ __forceinline__ Work work_of(const Product& g, uint32_t w) {
  const uint32_t tiles = g.tiles_m * g.tiles_n, split = w / tiles, t = w - split * tiles;
  const uint32_t tm = g.m_first ? t % g.tiles_m : t / g.tiles_n, tn = g.m_first ? t / g.tiles_m : t % g.tiles_n;
  Work r;
  r.m0 = tm * kTileM, r.n0 = tn * kTileN, r.split = split;
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

// What becomes of a warp's 32 rows and 128 columns of a finished tile
template <int EPI, class T>
__device__ __forceinline__ void finish_tile(const Product& g, const Work& w, uint32_t tensor, uint32_t half, uint32_t quarter, uint32_t lane, uint32_t* stage) {
  const uint32_t row = w.m0 + quarter * 32 + lane;
  const bool there = row < g.m;
  float v[32];
  if constexpr (EPI == kStats) {
    const int64_t target = there ? target_of(g.targets, g.token_bytes, row) - g.col0 : -1;
    float most = -CUDART_INF_F, sum = 0.0f;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (col >= g.n) break;
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = v[i] * g.k2;
      if (g.n - col < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (col + i >= g.n) v[i] = -CUDART_INF_F;
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
    if (there && w.n0 + half * 128 < g.n) g.stats[(uint64_t)(w.n0 / 128 + half) * g.stats_stride + row] = make_float2(most, sum);
  } else if constexpr (EPI == kProbs) {
    // x: ln sum exp in log2, less the exponent that is added; y: the weight, 0 where the row counts for nothing; z: the target's value
    const float4 r = there ? g.row[row] : make_float4(0, 0, 0, 0);
    const int64_t target = there ? target_of(g.targets, g.token_bytes, row) - g.col0 : -1;
    T* const out = static_cast<T*>(g.out) + (uint64_t)row * g.ldo;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (col >= g.n) break;
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
      if (there) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = pack2<T>(v[16 * h + 2 * i], v[16 * h + 2 * i + 1]);
          store_sector(out + col + 16 * h, p);
        }
      }
    }
  } else if constexpr (EPI == kParts) {
    float* const out = static_cast<float*>(g.out) + w.split * g.split_stride + (uint64_t)row * g.ldo;
    for (int c = 0; c < 4; ++c) {
      const uint32_t col = w.n0 + half * 128 + c * 32;
      if (col >= g.n) break;
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
      if (col >= g.n) break;
      tensor_load(tensor + c * 32, v);
      tensor_loaded(v);
      uint32_t p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = pack2<T>(v[2 * i] * alpha, v[2 * i + 1] * alpha);
      if (g.wide && col + 32 <= g.n) {
        if (there) {
          store_sector(out + (uint64_t)row * g.ldo + col, p);
          store_sector(out + (uint64_t)row * g.ldo + col + 16, p + 8);
        }
      } else {  // rows that begin anywhere: turned in shared memory, so that a warp writes neighbours
#pragma unroll
        for (int i = 0; i < 16; ++i) stage[lane * 17 + i] = p[i];
        __syncwarp();
        const uint16_t* const from = reinterpret_cast<const uint16_t*>(stage) + lane;
        uint16_t* const to = reinterpret_cast<uint16_t*>(out) + (uint64_t)(w.m0 + quarter * 32) * g.ldo + col + lane;
        const uint32_t rows = min(32u, g.m - min(g.m, w.m0 + quarter * 32));
        if (col + lane < g.n)
          for (uint32_t r = 0; r < rows; ++r) to[r * g.ldo] = from[r * 34];
        __syncwarp();
      }
    }
  }
}

template <int EPI, bool A_ROWS, bool B_ROWS, class T>
__global__ void __launch_bounds__(kThreads, 1) k_head_product(const __grid_constant__ Product g) {
  extern __shared__ uint8_t dynamic[];
  __shared__ uint64_t full[kStages], empty[kStages], made[2], taken[2], over;
  __shared__ uint32_t tensor_at, late;
  __shared__ uint32_t turn[EPI == kGrad ? kOutWarps * 32 * 17 : 1];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const uint32_t ring = (smem_at(dynamic) + 1023) & ~1023u;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 1);
    for (int i = 0; i < 2; ++i) mbar_init(made + i, 1), mbar_init(taken + i, kOutWarps);
    mbar_init(&over, 1);
    late = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tensor_alloc<1>(&tensor_at);
  tensor_before();
  __syncthreads();
  tensor_after();
  const uint32_t tensor = tensor_at, items = g.tiles_m * g.tiles_n * g.splits;
  pdl_enter();
  bool ok = true;
  if (warp == 0 && lane == 0) {
    uint32_t s = 0, phase = 0, issued = 0;
    for (uint32_t w = blockIdx.x; ok && w < items; w += gridDim.x) {
      const Work r = work_of(g, w);
      for (uint32_t k = r.k_from; k < r.k_to; ++k) {
        if (!(ok = mbar_wait(empty + s, phase ^ 1, &late))) break;
        mbar_expect(full + s, kBytesA + kBytesB);
        const uint32_t a = ring + s * (kBytesA + kBytesB), b = a + kBytesA, bar = smem_at(full + s);
        if constexpr (A_ROWS) {
#pragma unroll
          for (uint32_t i = 0; i < kTileM / 64; ++i) load_tile<1>(g.a, a + i * kTileBytes64, bar, r.m0 + 64 * i, k * kTileK);
        } else {
          load_tile<1>(g.a, a, bar, k * kTileK, r.m0);
        }
        if constexpr (B_ROWS) {
#pragma unroll
          for (uint32_t i = 0; i < kTileN / 64; ++i) load_tile<1>(g.b, b + i * kTileBytes64, bar, r.n0 + 64 * i, k * kTileK);
        } else {
          load_tile<1>(g.b, b, bar, k * kTileK, r.n0);
        }
        ++issued;
        if (++s == kStages) s = 0, phase ^= 1;
      }
    }
    if (!ok) {  // copies that are on their way end before the block does
      uint32_t none = 0;
      for (uint32_t i = 0; i < (issued < kStages ? issued : kStages); ++i) {
        if (s == 0) s = kStages, phase ^= 1;
        --s;
        mbar_wait(full + s, phase, &none, kMostWait / 4);
      }
    }
  } else if (warp == 1 && lane == 0) {
    constexpr uint32_t kind = product_kind(std::is_same<T, __nv_bfloat16>::value, A_ROWS, B_ROWS, kTileM, kTileN);
    uint32_t s = 0, phase = 0, turn_of = 0;
    bool any = false;
    for (uint32_t w = blockIdx.x; ok && w < items; w += gridDim.x, ++turn_of) {
      const Work r = work_of(g, w);
      const uint32_t half = turn_of & 1;
      if (!(ok = mbar_wait(taken + half, (turn_of / 2 & 1) ^ 1, &late))) break;
      tensor_after();
      for (uint32_t k = r.k_from; k < r.k_to; ++k) {
        if (!(ok = mbar_wait(full + s, phase, &late))) break;
        tensor_after();
        const uint32_t a = ring + s * (kBytesA + kBytesB), b = a + kBytesA;
#pragma unroll
        for (uint32_t i = 0; i < kTileK / 16; ++i)
          multiply<1>(tensor + half * kTileN, operand<A_ROWS>(a + i * kStepBytes<A_ROWS>), operand<B_ROWS>(b + i * kStepBytes<B_ROWS>), kind,
                      k != r.k_from || i != 0);
        commit<1>(empty + s);
        any = true;
        if (++s == kStages) s = 0, phase ^= 1;
      }
      if (ok) commit<1>(made + half);
    }
    if (!ok && any) {
      uint32_t none = 0;
      commit<1>(&over);
      mbar_wait(&over, 0, &none, kMostWait / 4);
    }
  } else if (warp >= 4) {
    const uint32_t half_tile = (warp - 4) / 4, quarter = warp & 3;
    uint32_t turn_of = 0;
    for (uint32_t w = blockIdx.x; w < items; w += gridDim.x, ++turn_of) {
      const Work r = work_of(g, w);
      const uint32_t half = turn_of & 1;
      if (!(ok = __all_sync(kFull, mbar_wait(made + half, turn_of / 2 & 1, &late)))) break;
      tensor_after();
      finish_tile<EPI, T>(g, r, tensor + half * kTileN + half_tile * 128 + (quarter * 32 << 16), half_tile, quarter, lane, turn + (EPI == kGrad ? (warp - 4) * 32 * 17 : 0));
      tensor_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(taken + half);
    }
  }
  __syncwarp();
  tensor_before();
  __syncthreads();
  tensor_after();
  if (warp == 2) tensor_free<1>(tensor);
  if (threadIdx.x == 0 && late) {
    *g.late = 1;
    if (g.status) set_status(g.status, CVLC_ERR_DEVICE_TIMEOUT);
  }
}

// ---- what is around them -------------------------------------------------------------------

struct Header {  // at the beginning of the workspace
  int32_t late;
  uint32_t largest;  // bits of the largest weight's size
  float up, down;    // a power of two that brings weights to at most 1, times 2^15 (fp16), and its inverse
};

// One block: what the call's kernels share
__global__ void __launch_bounds__(1024) k_head_begin(Header* h, const float* weight, const void* targets, uint32_t token_bytes, uint64_t rows, uint32_t vocab,
                                                     int half, int32_t* status) {
  __shared__ uint32_t most;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  uint32_t m = 0;
  bool beyond = false;
  for (uint64_t i = threadIdx.x; i < rows; i += blockDim.x) {
    const int64_t t = target_of(targets, token_bytes, i);
    if (t >= (int64_t)vocab) beyond = true;
    if (weight && t >= 0 && t < (int64_t)vocab) {
      const uint32_t w = __float_as_uint(weight[i]) & 0x7FFFFFFFu;
      if (w < 0x7F800000u) m = max(m, w);
    }
  }
  if (beyond && status) set_status(status, CVLC_ERR_INVALID_ARG);
  m = __reduce_max_sync(kFull, m);
  if ((threadIdx.x & 31) == 0) atomicMax(&most, m);
  __syncthreads();
  if (threadIdx.x == 0) {
    h->late = 0;
    // fp16 holds 2^-24 to 2^16: G, at most the largest weight in size, is held times a power of two that makes it at most 2^15
    const int e = !half ? 0 : weight ? (most ? min(max((int)(most >> 23) - 126, -100), 100) : 0) - 15 : -15;
    h->up = exp2f((float)-e), h->down = exp2f((float)e);
  }
}

// Rows of any alignment, copied to rows on 16 bytes, a warp each.  Rows that count for nothing become zeros: their values, which may be no numbers, have a part
// in the products of others' gradients.
__global__ void __launch_bounds__(256) k_head_align(const uint16_t* from, uint64_t from_stride, uint16_t* to, uint64_t to_stride, uint64_t rows, uint32_t dim,
                                                    const void* targets, uint32_t token_bytes, uint32_t vocab, const float* weight) {
  const uint64_t row = (uint64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const uint32_t lane = threadIdx.x & 31;
  if (row >= rows) return;
  const uint16_t* const src = from + row * from_stride;
  uint16_t* const dst = to + row * to_stride;
  bool counts = true;
  if (targets) {
    const int64_t t = target_of(targets, token_bytes, row);
    counts = t >= 0 && t < (int64_t)vocab && !(weight && weight[row] == 0.0f);
  }
  const bool vectors = reinterpret_cast<uintptr_t>(src) % 16 == 0;
  for (uint32_t i = lane * 8; i < dim; i += 256) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (counts) {
      if (vectors && i + 8 <= dim) {
        v = __ldg(reinterpret_cast<const uint4*>(src + i));
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

struct RowsArgs {
  const float2* stats;
  uint64_t stats_stride;
  uint32_t slots, token_bytes, vocab;
  const float* at_target;
  const void* targets;
  const float* weight;
  float* loss;
  float4* row;  // or nullptr
  const Header* header;
  uint64_t rows;
};
// A row's parts joined: 32 rows a block, eight threads a row.
// Sums relative to the largest; that of the words other than the target (o) is kept apart, so that 1 - q and a small loss ln(1 + o) keep their accuracy.
__global__ void __launch_bounds__(256) k_head_rows(const RowsArgs a) {
  pdl_enter();
  __shared__ float2 part[8][32];
  const uint32_t lane = threadIdx.x & 31, group = threadIdx.x / 32;
  const uint64_t row = (uint64_t)blockIdx.x * 32 + lane;
  float m = -CUDART_INF_F, s = 0.0f;
  if (row < a.rows) {
#pragma unroll 4
    for (uint32_t i = group; i < a.slots; i += 8) {
      const float2 x = a.stats[(uint64_t)i * a.stats_stride + row];
      const float n = fmaxf(m, x.x), from = n == -CUDART_INF_F ? 0.0f : n;
      s = s * exp2f(m - from) + x.y * exp2f(x.x - from);
      m = n;
    }
  }
  part[group][lane] = make_float2(m, s);
  __syncthreads();
  if (group || row >= a.rows) return;
  const int64_t target = target_of(a.targets, a.token_bytes, row);
  const float weight = a.weight ? a.weight[row] : 1.0f;
  if (target < 0 || target >= (int64_t)a.vocab || weight == 0.0f) {
    a.loss[row] = a.header->late ? CUDART_NAN_F : 0.0f;
    if (a.row) a.row[row] = make_float4(0, 0, 0, 0);
    return;
  }
  const float zt = a.at_target[row];
  float most = zt;
  for (int i = 0; i < 8; ++i) most = fmaxf(most, part[i][lane].x);
  double others = 0.0;
  for (int i = 0; i < 8; ++i)
    if (part[i][lane].x != -CUDART_INF_F || part[i][lane].y != 0.0f) others += (double)(part[i][lane].y * exp2f(part[i][lane].x - most));
  const float o = (float)others, right = exp2f(zt - most), total = right + o;
  const float loss = most == zt ? log1pf(o) : logf(total) + (most - zt) * kLn2;
  a.loss[row] = a.header->late ? CUDART_NAN_F : weight * loss;
  if (a.row) {
    const float w = weight * a.header->up;
    a.row[row] = make_float4(most + log2f(total), w, -(o / total) * w, 0.0f);
  }
}

struct JoinArgs {
  const float* parts;
  uint64_t split_stride, ldp, ldo;
  uint32_t splits, dim;
  uint64_t rows;
  float alpha;
  const Header* header;
  void* out;
};
template <class T>
__global__ void __launch_bounds__(256) k_head_join(const JoinArgs a) {
  pdl_enter();
  const float alpha = a.header->late ? CUDART_NAN_F : a.alpha * a.header->down;
  const uint32_t per = (a.dim + 3) / 4;
  const uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x, row = i / per;
  const uint32_t col = (uint32_t)(i - row * per) * 4;
  if (row >= a.rows) return;
  float4 s = make_float4(0, 0, 0, 0);
  for (uint32_t k = 0; k < a.splits; ++k) {
    const float4 x = *reinterpret_cast<const float4*>(a.parts + k * a.split_stride + row * a.ldp + col);
    s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
  }
  T* const out = static_cast<T*>(a.out) + row * a.ldo + col;
  const float v[4] = {s.x * alpha, s.y * alpha, s.z * alpha, s.w * alpha};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (col + k < a.dim) out[k] = from_float<T>(v[k]);
}

// ---- layout and launching --------------------------------------------------------------------

struct HeadLayout {
  bool copy_hidden, copy_head;
  uint64_t ld;  // of copies
  uint32_t piece, pieces;  // words
  uint64_t ldg, ldp, stats_stride;
  uint32_t splits;
  size_t off_hidden, off_head, off_stats, off_target, off_row, off_g, off_parts, total;
};
bool on16(const void* p, uint64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; }
uint32_t tiles(uint64_t n, uint32_t tile) { return (uint32_t)((n + tile - 1) / tile); }

// In how many parts a sum is cut: as many as leave the SMs the least to do one behind the other (a part more costs its reading and writing).
uint32_t splits_of(uint32_t tiles_all, uint32_t k_blocks) {
  uint32_t best = 1;
  double cost = 1e30;
  for (uint32_t s = 1; s <= 32 && s * 8 <= (k_blocks > 8 ? k_blocks : 8); ++s) {
    const double c = (double)((tiles_all * s + kNumSM - 1) / kNumSM) / s * k_blocks + 2.0 * s;
    if (c < cost * 0.98) cost = c, best = s;
  }
  return best;
}

HeadLayout head_layout(const cvlc_head& a, uint32_t pieces) {
  HeadLayout L = {};
  L.copy_hidden = pieces || !on16(a.hidden_dev, a.hidden_stride), L.copy_head = !on16(a.head_dev, a.head_stride);
  L.ld = (a.dim + 7) / 8 * 8;
  L.stats_stride = (a.rows + 31) / 32 * 32;
  size_t at = 256;
  auto take = [&](size_t bytes) { const size_t from = at; at = align256(at + bytes); return from; };
  L.off_hidden = take(L.copy_hidden ? a.rows * L.ld * 2 : 0);
  L.off_head = take(L.copy_head ? a.vocab * L.ld * 2 : 0);
  L.off_stats = take((size_t)tiles(a.vocab, 128) * L.stats_stride * 8);
  L.off_target = take(a.rows * 4);
  if (pieces) {
    L.piece = tiles((a.vocab + pieces - 1) / pieces, kTileN) * kTileN;
    L.pieces = tiles(a.vocab, L.piece);
    if (L.pieces == 1) L.piece = a.vocab;
    L.ldg = (L.piece + 31) / 32 * 32;
    L.ldp = (a.dim + 31) / 32 * 32;
    L.splits = splits_of(tiles(a.rows, kTileM) * tiles(a.dim, kTileN), tiles(L.piece, kTileK));
    L.off_row = take(a.rows * 16);
    L.off_g = take(a.rows * L.ldg * 2);
    L.off_parts = take((size_t)L.splits * a.rows * L.ldp * 4);
  }
  L.total = at;
  return L;
}

template <int EPI, bool A_ROWS, bool B_ROWS, class T>
cudaError_t run_product(int id, Product& g, cudaStream_t st) {
  static OncePerDevice once;
  const cudaError_t e = once_per_device(once, [] { return allow_shared(k_head_product<EPI, A_ROWS, B_ROWS, T>, kGemmShared); });
  if (e != cudaSuccess) return e;
  g.tiles_m = tiles(g.m, kTileM), g.tiles_n = tiles(g.n, kTileN);
  // the operand with more tiles is read once, the other one's stay in the L2 cache
  g.m_first = g.tiles_m <= g.tiles_n;
  const uint64_t items = (uint64_t)g.tiles_m * g.tiles_n * g.splits;
  launch_kernel(id, k_head_product<EPI, A_ROWS, B_ROWS, T>, dim3((uint32_t)(items < kNumSM ? items : kNumSM)), dim3(kThreads), kGemmShared, st, true, g);
  return cudaGetLastError();
}

template <class T>
cudaError_t run_head(const cvlc_head& a, uint32_t pieces, float* loss, void* d_hidden, uint64_t d_hidden_stride, void* d_head, uint64_t d_head_stride,
                     void* ws, cudaStream_t st) {
  constexpr bool bf16 = std::is_same<T, __nv_bfloat16>::value;
  const HeadLayout L = head_layout(a, pieces);
  uint8_t* const base = static_cast<uint8_t*>(ws);
  Header* const header = reinterpret_cast<Header*>(base);
  launch_kernel(kKHeadBegin, k_head_begin, dim3(1), dim3(a.rows > 256 ? 1024 : 256), 0, st, false, header, a.row_weight_dev, a.targets_dev, a.token_bytes,
                a.rows, a.vocab, bf16 ? 0 : 1, a.status_dev);
  const void *hidden = a.hidden_dev, *head = a.head_dev;
  uint64_t hidden_ld = a.hidden_stride, head_ld = a.head_stride;
  auto copy = [&](const void*& x, uint64_t& ld, uint64_t rows, size_t off, const void* targets) {
    launch_kernel(kKHeadAlign, k_head_align, dim3(tiles(rows, 8)), dim3(256), 0, st, false, static_cast<const uint16_t*>(x), ld,
                  reinterpret_cast<uint16_t*>(base + off), L.ld, rows, a.dim, targets, a.token_bytes, a.vocab, a.row_weight_dev);
    x = base + off, ld = L.ld;
  };
  if (L.copy_hidden) copy(hidden, hidden_ld, a.rows, L.off_hidden, a.targets_dev);
  if (L.copy_head) copy(head, head_ld, a.vocab, L.off_head, nullptr);

  Product p = {};
  p.m = (uint32_t)a.rows, p.n = a.vocab, p.k_blocks = tiles(a.dim, kTileK), p.splits = 1;
  p.k2 = a.scale * kLog2E, p.targets = a.targets_dev, p.token_bytes = a.token_bytes;
  p.stats = reinterpret_cast<float2*>(base + L.off_stats), p.stats_stride = L.stats_stride, p.at_target = reinterpret_cast<float*>(base + L.off_target);
  p.late = &header->late, p.status = a.status_dev;
  if (!make_tensor_map(&p.a, hidden, bf16, a.dim, a.rows, hidden_ld, kTileK, kTileM) || !make_tensor_map(&p.b, head, bf16, a.dim, a.vocab, head_ld, kTileK, kTileN))
    return cudaErrorUnknown;
  cudaError_t e = run_product<kStats, false, false, T>(kKHeadStats, p, st);
  if (e != cudaSuccess) return e;
  RowsArgs r = {};
  r.stats = p.stats, r.stats_stride = L.stats_stride, r.slots = tiles(a.vocab, 128), r.token_bytes = a.token_bytes, r.vocab = a.vocab;
  r.at_target = p.at_target, r.targets = a.targets_dev, r.weight = a.row_weight_dev, r.loss = loss, r.header = header, r.rows = a.rows;
  r.row = pieces ? reinterpret_cast<float4*>(base + L.off_row) : nullptr;
  launch_kernel(kKHeadRows, k_head_rows, dim3(tiles(a.rows, 32)), dim3(256), 0, st, true, r);
  if (!pieces) return cudaGetLastError();

  T* const G = reinterpret_cast<T*>(base + L.off_g);
  for (uint32_t i = 0; i < L.pieces; ++i) {
    const uint32_t from = i * L.piece, words = i + 1 < L.pieces ? L.piece : a.vocab - from;
    const T* const head_piece = static_cast<const T*>(head) + (uint64_t)from * head_ld;
    Product q = p;
    q.n = words, q.col0 = from, q.row = r.row, q.out = G, q.ldo = L.ldg;
    if (!make_tensor_map(&q.b, head_piece, bf16, a.dim, words, head_ld, kTileK, kTileN)) return cudaErrorUnknown;
    if ((e = run_product<kProbs, false, false, T>(kKHeadProbs, q, st)) != cudaSuccess) return e;
    q = Product{};
    q.late = p.late, q.status = p.status;
    q.m = (uint32_t)a.rows, q.n = a.dim, q.k_blocks = tiles(words, kTileK);
    q.splits = L.splits <= q.k_blocks ? L.splits : q.k_blocks;
    q.out = base + L.off_parts, q.ldo = L.ldp, q.split_stride = a.rows * L.ldp, q.add = i != 0;
    if (!make_tensor_map(&q.a, G, bf16, words, a.rows, L.ldg, kTileK, kTileM) || !make_tensor_map(&q.b, head_piece, bf16, a.dim, words, head_ld, 64, kTileK))
      return cudaErrorUnknown;
    if ((e = run_product<kParts, false, true, T>(kKHeadParts, q, st)) != cudaSuccess) return e;
    q = Product{};
    q.late = p.late, q.status = p.status;
    q.m = words, q.n = a.dim, q.k_blocks = tiles(a.rows, kTileK), q.splits = 1;
    T* const out = static_cast<T*>(d_head) + (uint64_t)from * d_head_stride;
    q.out = out, q.ldo = d_head_stride, q.wide = reinterpret_cast<uintptr_t>(out) % 32 == 0 && d_head_stride % 16 == 0;
    q.alpha = a.scale, q.alpha_dev = &header->down;
    if (!make_tensor_map(&q.a, G, bf16, words, a.rows, L.ldg, 64, kTileK) || !make_tensor_map(&q.b, hidden, bf16, a.dim, a.rows, hidden_ld, 64, kTileK))
      return cudaErrorUnknown;
    if ((e = run_product<kGrad, true, true, T>(kKHeadGrad, q, st)) != cudaSuccess) return e;
  }
  JoinArgs j = {};
  j.parts = reinterpret_cast<const float*>(base + L.off_parts), j.split_stride = a.rows * L.ldp, j.ldp = L.ldp, j.ldo = d_hidden_stride;
  j.splits = L.splits, j.dim = a.dim, j.rows = a.rows, j.alpha = a.scale, j.header = header, j.out = d_hidden;
  launch_kernel(kKHeadJoin, k_head_join<T>, dim3((uint32_t)((a.rows * ((a.dim + 3) / 4) + 255) / 256)), dim3(256), 0, st, true, j);
  return cudaGetLastError();
}

}  // namespace

size_t head_ws_bytes(const cvlc_head& a, uint32_t pieces) { return head_layout(a, pieces).total; }

cudaError_t launch_head(const cvlc_head& a, uint32_t pieces, float* loss, void* d_hidden, uint64_t d_hidden_stride, void* d_head, uint64_t d_head_stride, void* ws,
                        cudaStream_t st) {
  if (a.dtype == CVLC_F16) return run_head<__half>(a, pieces, loss, d_hidden, d_hidden_stride, d_head, d_head_stride, ws, st);
  return run_head<__nv_bfloat16>(a, pieces, loss, d_hidden, d_hidden_stride, d_head, d_head_stride, ws, st);
}

}  // namespace cvlc
