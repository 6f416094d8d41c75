// Rows of logits: what a client or a teacher answers (the top logits of every row) and distillation from such answers, the loss
// and its gradient.  A row's softmax needs its maximum and its sum of exponentials before anything can be written, so a row is
// cut over the blocks of a cluster, every thread keeps the 16-byte vectors that it has loaded in registers, the blocks exchange a
// few numbers through the cluster's shared memory, and the second half works from the registers: the logits are read once.
#include <cooperative_groups.h>

#include "cvlc_vocab.cuh"

namespace cg = cooperative_groups;

namespace cvlc {

namespace {

constexpr int kRowThreads = 512;  // most threads of a block

// ---- a row, cut into vectors and dealt to the blocks of a cluster --------------------------
// Vectors are aligned to 16 bytes in memory, so a row's first and last one may hold elements of other rows or none at all: those
// two are loaded and stored by elements.  Tiles of 32 vectors (a warp's load) go to the blocks in turn.  Vocabularies are often
// sorted by frequency: contiguous shares would leave the large logits to one block.
template <class T>
struct Row {
  const T* at;        // element 0
  uint32_t lead;      // elements of vector 0 that lie before it
  uint32_t vocab, vecs;
  uint32_t log_blocks, rank;

  __device__ __forceinline__ Row(const void* logits, uint64_t row, uint64_t stride, uint32_t vocab_, uint32_t log_blocks_, uint32_t rank_)
      : at(static_cast<const T*>(logits) + row * stride), vocab(vocab_), log_blocks(log_blocks_), rank(rank_) {
    lead = (uint32_t)((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(T));
    vecs = (lead + vocab + kPerVec<T> - 1) / kPerVec<T>;
  }
  // vectors of this block, in whole tiles
  __device__ __forceinline__ uint32_t share() const {
    const uint32_t tiles = (vecs + 31) >> 5, blocks = 1u << log_blocks;
    return ((tiles + blocks - 1 - rank) >> log_blocks) << 5;
  }
  // the block's i-th vector among the row's
  __device__ __forceinline__ uint32_t vec(uint32_t i) const { return ((((i >> 5) << log_blocks) | rank) << 5) | (i & 31); }
  // where this block has word j: the place among its elements, or -1
  __device__ __forceinline__ int place(uint32_t j) const {
    const uint32_t e = j + lead, v = e / kPerVec<T>, tile = v >> 5;
    if ((tile & ((1u << log_blocks) - 1)) != rank) return -1;
    return (int)((((tile >> log_blocks) << 5) | (v & 31)) * kPerVec<T> + e % kPerVec<T>);
  }
  // first word of a vector; below zero in the row's first one
  __device__ __forceinline__ int word(uint32_t v) const { return (int)(v * kPerVec<T>) - (int)lead; }
  __device__ __forceinline__ bool whole(uint32_t v) const {
    const int w = word(v);
    return w >= 0 && w + kPerVec<T> <= (int)vocab;
  }
  __device__ __forceinline__ uint4 load(uint32_t v) const {
    const int w = word(v);
    if (whole(v)) return __ldcs(reinterpret_cast<const uint4*>(at + w));
    float f[kPerVec<T>];
#pragma unroll
    for (int e = 0; e < kPerVec<T>; ++e) f[e] = (w + e >= 0 && w + e < (int)vocab) ? to_float(at[w + e]) : -CUDART_INF_F;
    return narrow<T>(f);
  }
};

// largest element of a vector; NaN only where all are
template <class T>
__device__ __forceinline__ float vec_max(const uint4& raw) {
  if constexpr (std::is_same<T, float>::value) {
    return fmaxf(fmaxf(__uint_as_float(raw.x), __uint_as_float(raw.y)), fmaxf(__uint_as_float(raw.z), __uint_as_float(raw.w)));
  } else {
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    T2 a, b, c, d;
    memcpy(&a, &raw.x, 4), memcpy(&b, &raw.y, 4), memcpy(&c, &raw.z, 4), memcpy(&d, &raw.w, 4);
    const T2 m = __hmax2(__hmax2(a, b), __hmax2(c, d));
    return fmaxf(to_float(m.x), to_float(m.y));
  }
}

// sum of exp((z - max) / temperature) relative to its own largest logit; max = -inf, sum = 0: nothing
struct MaxSum {
  float max, sum;
};
__device__ __forceinline__ float finite_ref(float m) { return m == -CUDART_INF_F ? 0.f : m; }
__device__ __forceinline__ MaxSum join(const MaxSum& a, const MaxSum& b, float c2) {
  const float m = fmaxf(a.max, b.max), ref = finite_ref(m);
  return {m, a.sum * exp2_fast((a.max - ref) * c2) + b.sum * exp2_fast((b.max - ref) * c2)};
}
__device__ __forceinline__ MaxSum warp_join(MaxSum a, float c2) {
#pragma unroll
  for (int o = 16; o; o >>= 1) a = join(a, {__shfl_xor_sync(kFull, a.max, o), __shfl_xor_sync(kFull, a.sum, o)}, c2);
  return a;
}

// The differences z - max are taken before the scaling by log2(e) / temperature: with rows masked by the type's lowest value, or far
// from zero, the product alone would overflow or lose the difference.
template <class T, int NV>
__device__ __forceinline__ void add_batch(const uint4 (&raw)[NV], float c2, MaxSum& acc) {
  float m = acc.max;
#pragma unroll
  for (int j = 0; j < NV; ++j) m = fmaxf(m, vec_max<T>(raw[j]));
  const float ref = finite_ref(m);
  float sum = acc.sum * exp2_fast((acc.max - ref) * c2);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float f[kPerVec<T>];
    widen<T>(raw[j], f);
    float part = 0.f;
#pragma unroll
    for (int e = 0; e < kPerVec<T>; ++e) part += exp2_fast((f[e] - ref) * c2);
    sum += part;
  }
  acc = {m, sum};
}

// ---- distillation ---------------------------------------------------------------------------
//
// z the student's logits over a vocabulary of V words, it = 1 / temperature, q = softmax(z it);
// the teacher's records (word, log-probability) give p_j = the sum of exp(logp) over the records of word j, P = sum p.
//   none    L = sum p_j (ln p_j - ln q_j)                              dL/dz_j = it (P q_j - p_j)
//   scaled  the same of p / P
//   bucket  with pr = max(0, 1 - P) and qr = the sum of q over the words that are not listed
//           L + pr (ln pr - ln qr)      dL/dz_j = it ((P + pr) q_j - p_j), not listed: it ((P + pr) q_j - pr q_j / qr)
// The listed and the unlisted words have sums of their own: qr may be far below what 1 - sum q can hold in 32 bits, and the listed
// words' gradients are written on their own anyway (by the threads that hold the records, behind the vectors).  Relative to the
// unlisted words' own maximum r the gradient of an unlisted word is one exponential and one product:
//   it exp((z_j - r) it) A,  A = (P + pr) exp((r - m) it) / s - pr / s_r.
// A block marks the listed words of its share in a bitmap in shared memory, where a second record of a word is noticed too.
// The teacher's sums are a few numbers a row and are held in 64 bits: what a list leaves over is often a small difference from one.

struct Said {  // listed words: their exponentials, and the sums of p, p ln p and p (z - all.max)
  MaxSum all;
  double mass, ent, cross;
};
// what p (z - a) has to gain to be p (z - b), a at most b; a = -inf: it is -inf already, or there is no mass
__device__ __forceinline__ double moved(double mass, float a, float b) {
  return a == -CUDART_INF_F || a == b ? 0.0 : mass * ((double)a - (double)b);
}
__device__ __forceinline__ Said join(const Said& a, const Said& b, float c2) {
  const MaxSum all = join(a.all, b.all, c2);
  return {all, a.mass + b.mass, a.ent + b.ent, (a.cross + moved(a.mass, a.all.max, all.max)) + (b.cross + moved(b.mass, b.all.max, all.max))};
}
__device__ __forceinline__ Said warp_join(Said a, float c2) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Said b = {{__shfl_xor_sync(kFull, a.all.max, o), __shfl_xor_sync(kFull, a.all.sum, o)},
                    __shfl_xor_sync(kFull, a.mass, o), __shfl_xor_sync(kFull, a.ent, o), __shfl_xor_sync(kFull, a.cross, o)};
    a = join(a, b, c2);
  }
  return a;
}
// one listed word of probability p with ln p, and its logit
__device__ __forceinline__ Said said_of(double p, double ln_p, float z) {
  const bool masked = z == -CUDART_INF_F;
  return {{z, masked ? 0.f : 1.f}, p, p != 0.0 ? p * ln_p : 0.0, masked && p != 0.0 ? -p * CUDART_INF : 0.0};
}
struct Part {  // a block's share of a row
  MaxSum rest;  // unlisted words
  Said said;
};
__device__ __forceinline__ Part join(const Part& a, const Part& b, float c2) { return {join(a.rest, b.rest, c2), join(a.said, b.said, c2)}; }
struct Whole {  // what the row's gradient needs; kept for it between loss and gradient
  float ref, a;         // unlisted words: a exp((z - ref) it)
  float max, inv_sum;   // q = exp((z - max) it) inv_sum
  float b, c;           // listed words: b q - c p
};
static_assert(sizeof(Whole) <= 4 * CVLC_DISTILL_STATS, "a row's place in the buffer");

__device__ __forceinline__ Whole whole_row(const Part* parts, uint32_t blocks, uint32_t rest, float temperature, float c2, double* loss) {
  Part p = parts[0];
  for (uint32_t r = 1; r < blocks; ++r) p = join(p, parts[r], c2);
  const MaxSum un = p.rest;
  const double mass = p.said.mass;
  const MaxSum all = join(un, p.said.all, c2);
  if (all.max == -CUDART_INF_F && all.sum == 0.f) {  // every word is masked: no distribution, no loss
    *loss = 0.0;
    return {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  }
  const double it = 1.0 / (double)temperature;
  const double ln_sum = log((double)all.sum), cross = p.said.cross + moved(mass, p.said.all.max, all.max);
  Whole w;
  w.max = all.max;
  w.inv_sum = 1.f / all.sum;
  double b = mass, c = 1.0, left = 0.0;
  *loss = p.said.ent - cross * it + mass * ln_sum;
  if (rest == CVLC_REST_SCALED) {
    b = mass > 0.0 ? 1.0 : mass;  // (a NaN stays one)
    c = mass > 0.0 ? 1.0 / mass : mass;
    *loss = mass > 0.0 ? *loss * c - log(mass) : mass;
  }
  const bool some = !(un.max == -CUDART_INF_F && un.sum == 0.f);  // else the list holds every word that the student may say
  if (rest == CVLC_REST_BUCKET && some) {
    left = mass < 1.0 ? 1.0 - mass : 0.0;
    b = mass + left;
    if (left > 0.0) *loss += left * (log(left) - (((double)un.max - (double)all.max) * it + log((double)un.sum) - ln_sum));
  }
  w.b = (float)b;
  w.c = (float)c;
  w.ref = some ? un.max : 0.f;
  w.a = some ? (float)(b * (double)(exp2_fast((un.max - all.max) * c2) * w.inv_sum) - (left > 0.0 ? left / (double)un.sum : 0.0)) : 0.f;
  return w;
}

// bits of the listed words of the block's vector i
template <class T>
__device__ __forceinline__ uint32_t listed_of(const uint8_t* marks, uint32_t i) {
  return kPerVec<T> == 8 ? marks[i] : (marks[i >> 1] >> ((i & 1) * 4)) & 15u;
}

template <class T, int NV, DistillKind KIND>
__global__ void __launch_bounds__(kRowThreads, 2) k_distill(DistillArgs a, uint32_t log_blocks, uint32_t share_most) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Part parts[kMaxClusterBlocks];
  __shared__ Part of_warp[kRowThreads / 32];
  __shared__ Whole whole;
  const uint32_t nt = blockDim.x, tid = threadIdx.x, blocks = 1u << log_blocks;
  const uint32_t rank = blockIdx.x & (blocks - 1);
  const uint64_t row = blockIdx.x >> log_blocks;
  const Row<T> R(a.logits, row, a.row_stride, a.vocab, log_blocks, rank);
  const float weight = a.row_weight ? a.row_weight[row] : 1.f;
  const float c2 = (float)((double)1.4426950408889634074 / (double)a.temperature);
  const uint32_t share = R.share();

  uint8_t* const marks = dyn;
  const uint32_t mark_bytes = (share_most * kPerVec<T> / 8 + 15) & ~15u;
  int* const at = reinterpret_cast<int*>(dyn + mark_bytes);  // places of the records in the block's share, or -1
  float* const prob = reinterpret_cast<float*>(at + a.k);    // their probabilities; -1: counted with an earlier record of the word
  float* const logit = prob + a.k;                           // the student's logits of their words

  // a row that counts for nothing is not looked at (but for what a later gradient may ask for)
  const bool idle = weight == 0.f && !(KIND == kDistillLoss && a.stats);

  uint4 raw[NV];
  if (!idle) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint32_t i = tid + j * nt;
      raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
    }
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (KIND != kDistillGrad && blocks > 1) cluster.sync();  // the other blocks have begun: their shared memory may be written
  if (!idle) {
    for (uint32_t i = tid; i < mark_bytes / 4; i += nt) reinterpret_cast<uint32_t*>(marks)[i] = 0;
    __syncthreads();
    bool twice = false;
    for (uint32_t i = tid; i < a.k; i += nt) {
      const int id = a.ids[row * a.k + i];
      int p = -1;
      if (id >= 0 && (uint32_t)id >= a.vocab) {
        if (a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
      } else if (id >= 0 && (p = R.place((uint32_t)id)) >= 0) {
        logit[i] = to_float(R.at[id]);
        const uint32_t bit = 1u << (p & 31);
        twice |= (atomicOr(reinterpret_cast<uint32_t*>(marks) + (p >> 5), bit) & bit) != 0;
      }
      at[i] = p;
      prob[i] = a.logp[row * a.k + i];
    }
    twice = __syncthreads_or(twice);
    // p of every word, summed in the order of its records
    Part mine = {{-CUDART_INF_F, 0.f}, {{-CUDART_INF_F, 0.f}, 0.0, 0.0, 0.0}};
    for (uint32_t i = tid; i < a.k; i += nt) {
      double p = -1.0;
      if (at[i] >= 0) {
        const double lp = (double)prob[i];
        p = exp(lp);
        bool merged = false;
        if (twice) {
          const int here = at[i];
          for (uint32_t o = 0; o < i; ++o)
            if (at[o] == here) p = -1.0;
          if (p >= 0.0)
            for (uint32_t o = i + 1; o < a.k; ++o)
              if (at[o] == here) p += exp((double)a.logp[row * a.k + o]), merged = true;
        }
        if (KIND != kDistillGrad && !(p < 0.0)) mine.said = join(mine.said, said_of(p, merged ? log(p) : lp, logit[i]), c2);
      }
      prob[i] = (float)p;  // only this thread reads its own
    }
    if (KIND == kDistillGrad) {
      if (tid == 0) whole = *reinterpret_cast<const Whole*>(a.stats + row * CVLC_DISTILL_STATS);
    } else {
      for (uint32_t base = 0; base < share; base += NV * nt) {
        if (base) {
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            const uint32_t i = base + tid + j * nt;
            raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
          }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const uint32_t i = base + tid + j * nt;
          if (i < share)
            if (const uint32_t bits = listed_of<T>(marks, i)) drop_elements<T>(raw[j], bits);
        }
        add_batch<T, NV>(raw, c2, mine.rest);
      }
      mine.rest = warp_join(mine.rest, c2);
      mine.said = warp_join(mine.said, c2);
      if ((tid & 31) == 0) of_warp[tid >> 5] = mine;
      __syncthreads();
      if (tid < blocks) {  // thread r hands the block's sums to block r
        Part p = of_warp[0];
        for (uint32_t w = 1; w < nt / 32; ++w) p = join(p, of_warp[w], c2);
        *(blocks > 1 ? cluster.map_shared_rank(&parts[rank], tid) : &parts[rank]) = p;
      }
    }
  }
  if (KIND != kDistillGrad && blocks > 1) cluster.sync();
  if (KIND != kDistillGrad && tid == 0) {
    double loss = 0.0;
    if (!idle) whole = whole_row(parts, blocks, a.rest, a.temperature, c2, &loss);
    if (rank == 0) {
      a.loss[row] = weight == 0.f ? 0.f : (float)((double)weight * loss);
      if (KIND == kDistillLoss && a.stats) *reinterpret_cast<Whole*>(a.stats + row * CVLC_DISTILL_STATS) = whole;
    }
  }
  if (KIND == kDistillLoss) return;
  __syncthreads();

  // the gradient, a vector at a time; where logits and gradient lie differently against 16 bytes, by elements
  T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
  const bool alike = ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(R.at)) & 15) == 0;
  const Whole w = idle ? Whole{} : whole;
  const float scale = idle ? 0.f : weight / a.temperature;
  const float ca = w.a * scale;
  for (uint32_t base = 0; base < share; base += NV * nt) {
    if (!idle && share > NV * nt) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const uint32_t i = base + tid + j * nt;
        raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint32_t i = base + tid + j * nt;
      if (i >= share) continue;
      const uint32_t v = R.vec(i);
      if (v >= R.vecs) continue;
      float f[kPerVec<T>];
      if (idle) {
#pragma unroll
        for (int e = 0; e < kPerVec<T>; ++e) f[e] = 0.f;
      } else {
        widen<T>(raw[j], f);
#pragma unroll
        for (int e = 0; e < kPerVec<T>; ++e) f[e] = ca * exp2_fast((f[e] - w.ref) * c2);
      }
      const int word = R.word(v);
      if (alike && R.whole(v)) {
        *reinterpret_cast<uint4*>(g + word) = narrow<T>(f);
      } else {
#pragma unroll
        for (int e = 0; e < kPerVec<T>; ++e)
          if (word + e >= 0 && word + e < (int)R.vocab) g[word + e] = from_float<T>(f[e]);
      }
    }
  }
  if (idle) return;
  __syncthreads();  // the listed words' gradients replace what the vectors hold in their places
  const float cb = w.b * scale, cc = w.c * scale;
  for (uint32_t i = tid; i < a.k; i += nt)
    if (at[i] >= 0 && !(prob[i] < 0.f)) {
      const float q = exp2_fast((logit[i] - w.max) * c2) * w.inv_sum;
      g[a.ids[row * a.k + i]] = from_float<T>(cb * q - cc * prob[i]);
    }
}

// how a call's rows are cut: blocks of a cluster for each, threads of a block
struct Cut {
  uint32_t log_blocks, threads, share;  // share: most vectors of a block
};

Cut cut_rows(uint64_t rows, uint32_t vocab, uint32_t per_vec, uint32_t nv) {
  const uint32_t vecs = vocab / per_vec + 2, tiles = (vecs + 31) / 32;
  Cut c = {0, 0, 0};
  while (c.log_blocks < 3 && ((tiles + (1u << c.log_blocks) - 1) >> c.log_blocks) * 32 > nv * kRowThreads) ++c.log_blocks;
  while (c.log_blocks < 3 && (rows << c.log_blocks) < 2 * kNumSM && (vecs >> c.log_blocks) >= 512) ++c.log_blocks;
  c.share = ((tiles + (1u << c.log_blocks) - 1) >> c.log_blocks) * 32;
  uint32_t t = (c.share + nv - 1) / nv;
  t = (t + 31) & ~31u;
  c.threads = t < 64 ? 64 : (t > kRowThreads ? kRowThreads : t);
  return c;
}

template <class... Params, class... Args>
cudaError_t launch_rows(int id, void (*kernel)(Params...), uint64_t rows, const Cut& c, bool clusters, size_t smem, cudaStream_t st, Args&&... args) {
  if (smem > 40 * 1024) {
    const cudaError_t e = allow_shared(kernel, smem);
    if (e != cudaSuccess) return e;
  }
  LaunchScope ls(id, st);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows << c.log_blocks));
  cfg.blockDim = dim3(c.threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 1u << c.log_blocks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = clusters && c.log_blocks ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
  const cudaError_t last = cudaGetLastError();
  return e != cudaSuccess ? e : last;
}

template <class T, DistillKind KIND>
cudaError_t distill_typed(const DistillArgs& a, cudaStream_t st) {
  constexpr int NV = 8;
  const Cut c = cut_rows(a.rows, a.vocab, kPerVec<T>, NV);
  const size_t smem = ((c.share * kPerVec<T> / 8 + 15) & ~15u) + (size_t)a.k * 12;
  return launch_rows(KIND == kDistillLoss ? kKDistillLoss : KIND == kDistillGrad ? kKDistillGrad : kKDistillStep, k_distill<T, NV, KIND>, a.rows, c,
                     KIND != kDistillGrad, smem, st, a, c.log_blocks, c.share);
}
template <class T>
cudaError_t distill_kind(const DistillArgs& a, DistillKind kind, cudaStream_t st) {
  switch (kind) {
    case kDistillLoss: return distill_typed<T, kDistillLoss>(a, st);
    case kDistillGrad: return distill_typed<T, kDistillGrad>(a, st);
    default: return distill_typed<T, kDistillStep>(a, st);
  }
}

// ---- top logits --------------------------------------------------------------------------------
//
// The k largest logits of a row, in order, equal ones by ascending word; each with its log-probability.  Of the elements
// a thread has loaded, only the largest is looked at first: with `blocks` blocks a row, the ceil(k / blocks)-th largest of a block's
// thread maxima has that many elements at or above it, so the smallest of the blocks' bounds has at least k in the row, and
// hardly more (a thread rarely holds two).  What lies at or above it goes to the first block and is ranked there by (value, word).
// Rows with more such elements than the lists hold (whole rows of equal logits) are selected digit by digit instead.

constexpr uint32_t kTopList = 2048;  // candidates of a row

// floats in the order of unsigned numbers, zeros of either sign alike
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
constexpr uint32_t kOrderNegInf = 0x007FFFFFu;  // order_of(-inf); what is not above it is never listed
__device__ __forceinline__ unsigned long long candidate(uint32_t order, uint32_t word) {
  return ((unsigned long long)order << 32) | (uint32_t)~word;
}

struct TopPart {
  MaxSum all;
  uint32_t bound;
};

template <class T, int NV>
__global__ void __launch_bounds__(kRowThreads, 2) k_top_logits(TopArgs a, uint32_t log_blocks) {
  __shared__ unsigned long long list[kTopList];    // in the first block: a stretch for every block
  __shared__ unsigned long long packed[kTopList];  // the same without gaps
  __shared__ TopPart parts[kMaxClusterBlocks];
  __shared__ MaxSum of_warp[kRowThreads / 32];
  __shared__ uint32_t counts[kMaxClusterBlocks];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t mine, picked, above;
  __shared__ MaxSum of_block;
  const uint32_t nt = blockDim.x, tid = threadIdx.x, blocks = 1u << log_blocks;
  const uint32_t rank = blockIdx.x & (blocks - 1);
  const uint64_t row = blockIdx.x >> log_blocks;
  const Row<T> R(a.logits, row, a.row_stride, a.vocab, log_blocks, rank);
  const float c2 = (float)((double)1.4426950408889634074 / (double)a.temperature);
  const uint32_t share = R.share();
  cg::cluster_group cluster = cg::this_cluster();

  uint4 raw[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const uint32_t i = tid + j * nt;
    raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
  }
  if (tid == 0) mine = 0;
  if (blocks > 1) cluster.sync();

  MaxSum acc = {-CUDART_INF_F, 0.f};
  for (uint32_t base = 0; base < share; base += NV * nt) {
    if (base) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const uint32_t i = base + tid + j * nt;
        raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
      }
    }
    add_batch<T, NV>(raw, c2, acc);
  }
  const uint32_t top = order_of(acc.max);
  const MaxSum warp = warp_join(acc, c2);
  if ((tid & 31) == 0) of_warp[tid >> 5] = warp;
  __syncthreads();
  if (tid == 0) {
    MaxSum s = of_warp[0];
    for (uint32_t w = 1; w < nt / 32; ++w) s = join(s, of_warp[w], c2);
    of_block = s;
  }
  __syncthreads();
  // the largest bound that `want` threads reach, by halving
  const uint32_t want = (a.k + blocks - 1) >> log_blocks;
  uint32_t lo = kOrderNegInf + 1, hi = order_of(of_block.max);
  if ((uint32_t)__syncthreads_count(top >= lo) < want) hi = lo;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    if ((uint32_t)__syncthreads_count(top >= mid) >= want) lo = mid;
    else hi = mid - 1;
  }
  if (tid < blocks) *(blocks > 1 ? cluster.map_shared_rank(&parts[rank], tid) : &parts[rank]) = {of_block, lo};
  if (blocks > 1) cluster.sync();
  else __syncthreads();
  uint32_t bound = parts[0].bound;
  MaxSum all = parts[0].all;
  for (uint32_t r = 1; r < blocks; ++r) {
    bound = min(bound, parts[r].bound);
    all = join(all, parts[r].all, c2);
  }
  const bool spoiled = !(all.sum < CUDART_INF_F);  // a NaN or +inf among the logits: there is no softmax
  const uint32_t stretch = kTopList >> log_blocks;

  // elements from `least` on (a candidate: value and word) into the first block's list
  auto gather = [&](unsigned long long least) {
    unsigned long long* const to = (blocks > 1 ? cluster.map_shared_rank(list, 0) : list) + rank * stretch;
    const float floor_value = value_of((uint32_t)(least >> 32));
    for (uint32_t base = 0; base < share; base += NV * nt) {
      if (share > NV * nt) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const uint32_t i = base + tid + j * nt;
          raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
        }
      }
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (!(vec_max<T>(raw[j]) >= floor_value)) continue;
        const uint32_t i = base + tid + j * nt;
        float f[kPerVec<T>];
        widen<T>(raw[j], f);
        const int word = R.word(R.vec(i));
#pragma unroll
        for (int e = 0; e < kPerVec<T>; ++e) {
          const unsigned long long c = candidate(order_of(f[e]), (uint32_t)(word + e));
          if (f[e] >= floor_value && c >= least) {
            const uint32_t n = atomicAdd(&mine, 1u);
            if (n < stretch) to[n] = c;
          }
        }
      }
    }
    __syncthreads();
    if (tid < blocks) *(blocks > 1 ? cluster.map_shared_rank(&counts[rank], tid) : &counts[rank]) = mine;
    if (blocks > 1) cluster.sync();
    else __syncthreads();
  };
  bool overflow = false;
  if (!spoiled) {
    gather((unsigned long long)bound << 32);
    for (uint32_t r = 0; r < blocks; ++r) overflow |= counts[r] > stretch;
  }
  if (overflow) {
    // the k-th largest candidate, eight bits at a time
    unsigned long long prefix = 0;
    uint32_t left = a.k;  // rank of the wanted one among those that share the prefix
    for (int shift = 56; shift >= 0; shift -= 8) {
      for (uint32_t i = tid; i < 256; i += nt) hist[i] = 0;
      __syncthreads();
      uint32_t last = 0, run = 0;  // equal digits in a row are counted at once
      for (uint32_t base = 0; base < share; base += NV * nt) {
        if (share > NV * nt) {
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            const uint32_t i = base + tid + j * nt;
            raw[j] = R.load(i < share ? R.vec(i) : R.vecs);
          }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float f[kPerVec<T>];
          widen<T>(raw[j], f);
          const int word = R.word(R.vec(base + tid + j * nt));
#pragma unroll
          for (int e = 0; e < kPerVec<T>; ++e) {
            if (!(f[e] > -CUDART_INF_F)) continue;
            const unsigned long long c = candidate(order_of(f[e]), (uint32_t)(word + e));
            if (shift < 56 && (c >> (shift + 8)) != prefix) continue;
            const uint32_t digit = (uint32_t)(c >> shift) & 255u;
            if (run && digit != last) {
              atomicAdd(&hist[last], run);
              run = 0;
            }
            last = digit;
            ++run;
          }
        }
      }
      if (run) atomicAdd(&hist[last], run);
      if (blocks > 1) cluster.sync();
      else __syncthreads();
      if (tid < 32) {  // eight digits a lane, from the largest down
        uint32_t n[8], sum = 0;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          n[d] = 0;
          for (uint32_t r = 0; r < blocks; ++r) n[d] += (blocks > 1 ? cluster.map_shared_rank(hist, r) : hist)[255 - (tid * 8 + d)];
          sum += n[d];
        }
        uint32_t before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(kFull, before, o);
          if (tid >= (uint32_t)o) before += v;
        }
        before -= sum;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          if (before < left && left <= before + n[d]) picked = 255 - (tid * 8 + d), above = before;
          before += n[d];
        }
      }
      __syncthreads();
      prefix = (prefix << 8) | picked;
      left -= above;
      if (blocks > 1) cluster.sync();  // the counts have been read
      else __syncthreads();
    }
    if (tid == 0) mine = 0;
    __syncthreads();
    gather(prefix);
  }

  if (rank != 0) return;
  if (spoiled) {
    for (uint32_t i = tid; i < a.k; i += nt) {
      a.ids[row * a.k + i] = (int32_t)i;
      a.logp[row * a.k + i] = CUDART_NAN_F;
    }
    return;
  }
  uint32_t n = 0;
  for (uint32_t r = 0; r < blocks; ++r) {
    const uint32_t c = counts[r];
    for (uint32_t i = tid; i < c; i += nt) packed[n + i] = list[r * stretch + i];
    n += c;
  }
  __syncthreads();
  const double it = 1.0 / (double)a.temperature, ln_sum = log((double)all.sum);
  for (uint32_t i = tid; i < n; i += nt) {
    const unsigned long long c = packed[i];
    uint32_t larger = 0;
    for (uint32_t o = 0; o < n; ++o) larger += packed[o] > c;
    if (larger < a.k) {
      a.ids[row * a.k + larger] = (int32_t)~(uint32_t)c;
      a.logp[row * a.k + larger] = (float)(((double)value_of((uint32_t)(c >> 32)) - (double)all.max) * it - ln_sum);
    }
  }
  for (uint32_t i = n + tid; i < a.k; i += nt) {  // fewer words than records: the others are masked
    a.ids[row * a.k + i] = -1;
    a.logp[row * a.k + i] = -CUDART_INF_F;
  }
}

template <class T>
cudaError_t top_typed(const TopArgs& a, cudaStream_t st) {
  constexpr int NV = 8;
  const Cut c = cut_rows(a.rows, a.vocab, kPerVec<T>, NV);
  return launch_rows(kKTopLogits, k_top_logits<T, NV>, a.rows, c, true, 0, st, a, c.log_blocks);
}

}  // namespace

cudaError_t launch_top_logits(const TopArgs& a, uint32_t dtype, cudaStream_t st) {
  if (dtype == CVLC_F32) return top_typed<float>(a, st);
  if (dtype == CVLC_F16) return top_typed<__half>(a, st);
  return top_typed<__nv_bfloat16>(a, st);
}

cudaError_t launch_distill(const DistillArgs& a, uint32_t dtype, DistillKind kind, cudaStream_t st) {
  if (dtype == CVLC_F32) return distill_kind<float>(a, kind, st);
  if (dtype == CVLC_F16) return distill_kind<__half>(a, kind, st);
  return distill_kind<__nv_bfloat16>(a, kind, st);
}

}  // namespace cvlc
