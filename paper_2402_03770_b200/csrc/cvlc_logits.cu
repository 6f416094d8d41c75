// Rows of logits: what a client or a teacher answers (the top logits of every row) and distillation from such answers, the loss
// and its gradient.  All are bound by the reading of the logits (0.5 to 3 operations a byte, none of which a matrix instruction does) and, where
// rows are few or short, by the chain of load, maximum, sum, exchange and store.  A row's softmax needs its maximum and its sum of
// exponentials before anything can be written.
// Few or short rows: a row is cut over the blocks of a cluster, every thread keeps the 16-byte vectors that it has loaded in registers, the
// blocks exchange a few numbers through the cluster's shared memory, and the second half works from the registers: the logits are read once.
// Many long rows: two blocks an SM go from row to row, and what a row needs beside its elements is done by warps of their own.
// streamed() says which, with both sides' times.
#include <cooperative_groups.h>

#include "cvlc_vocab.cuh"

namespace cg = cooperative_groups;

namespace cvlc {

namespace {

constexpr int kRowThreads = 512;  // most threads of a block

// ---- a row, cut into vectors and dealt to the blocks of a cluster --------------------------
// Vectors are aligned to 16 bytes in memory, so a row's first and last one may hold elements of other rows or none at all: those
// two are loaded and stored by elements.  Tiles of 32 vectors (a warp's load) go to the warps of the cluster's blocks in turn, the blocks
// first: vocabularies are often sorted by frequency, and contiguous shares would leave the large logits to one block.  A thread's
// i-th vector is then vector first + i * apart of the row.
template <class T>
struct Row {
  const T* at;                 // word 0
  const uint4* from;           // vector 0
  uint32_t lead;               // elements of vector 0 that lie before word 0
  uint32_t vocab, vecs;
  uint32_t log_blocks, rank;
  uint32_t first, apart;       // of the thread
  uint32_t whole_from, wholes; // vectors whose elements are all the row's

  __device__ __forceinline__ Row(const void* logits, uint64_t row, uint64_t stride, uint32_t vocab_, uint32_t log_blocks_, uint32_t rank_)
      : at(static_cast<const T*>(logits) + row * stride), vocab(vocab_), log_blocks(log_blocks_), rank(rank_) {
    lead = (uint32_t)((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(T));
    from = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)15);
    vecs = (lead + vocab + kPerVec<T> - 1) / kPerVec<T>;
    whole_from = lead ? 1 : 0;
    const uint32_t whole_to = (lead + vocab) / kPerVec<T>;
    wholes = whole_to > whole_from ? whole_to - whole_from : 0;
    first = ((((threadIdx.x >> 5) << log_blocks) | rank) << 5) | (threadIdx.x & 31);
    apart = ((blockDim.x >> 5) << log_blocks) << 5;
  }
  // vectors that a thread of this block has at most
  __device__ __forceinline__ uint32_t rounds() const { return (vecs + apart - 1) / apart; }
  // where this block has word j: thread + block size * round, in elements, or -1
  __device__ __forceinline__ int place(uint32_t j) const {
    const uint32_t e = j + lead, v = e / kPerVec<T>, tile = v >> 5;
    if ((tile & ((1u << log_blocks) - 1)) != rank) return -1;
    return (int)((((tile >> log_blocks) << 5) | (v & 31)) * kPerVec<T> + e % kPerVec<T>);
  }
  // first word of a vector; below zero in the row's first one
  __device__ __forceinline__ int word(uint32_t v) const { return (int)(v * kPerVec<T>) - (int)lead; }
  __device__ __forceinline__ bool whole(uint32_t v) const { return v - whole_from < wholes; }
  __device__ __forceinline__ bool ragged() const { return wholes != vecs; }
  __device__ uint4 load_elements(uint32_t v) const {
    const int w = word(v);
    float f[kPerVec<T>];
#pragma unroll
    for (int e = 0; e < kPerVec<T>; ++e) f[e] = (w + e >= 0 && w + e < (int)vocab) ? to_float(at[w + e]) : -CUDART_INF_F;
    return narrow<T>(f);
  }
};

// all elements minus infinity
template <class T>
__device__ __forceinline__ uint4 nothing() {
  constexpr uint32_t w = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
  return make_uint4(w, w, w, w);
}

// rounds `from` .. from + NV - 1 of the thread; what lies behind the row is minus infinity
template <class T, int NV>
__device__ __forceinline__ void load_batch(const Row<T>& R, uint32_t from, uint4 (&raw)[NV]) {
  const uint32_t v0 = R.first + from * R.apart;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    raw[j] = nothing<T>();
    if (R.whole(v0 + j * R.apart)) raw[j] = __ldcs(R.from + v0 + j * R.apart);
  }
  if (R.ragged()) {  // the first and the last vector
    const uint32_t last = R.vecs - 1;
    const bool mine_first = !R.whole(0) && v0 == 0;
    const bool mine_last = !R.whole(last) && last && last >= v0 && (last - v0) % R.apart == 0 && (last - v0) / R.apart < NV;
    if (mine_first) raw[0] = R.load_elements(0);
    if (mine_last) {
      const uint4 r = R.load_elements(last);
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (v0 + j * R.apart == last) raw[j] = r;
    }
  }
}

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
// over the lanes of a warp: the maximum first, then every sum is moved to it once
__device__ __forceinline__ MaxSum warp_join(const MaxSum& a, float c2) {
  float m = a.max;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
  float s = a.sum * exp2_fast((a.max - finite_ref(m)) * c2);
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  return {m, s};
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
  return v;
}
template <class V>
__device__ __forceinline__ V warp_sum(V v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}
// over what the first `n` lanes read from an array of the warps
__device__ __forceinline__ MaxSum join_warps(const MaxSum* of_warp, uint32_t n, float c2) {
  const uint32_t lane = threadIdx.x & 31;
  return warp_join(lane < n ? of_warp[lane] : MaxSum{-CUDART_INF_F, 0.f}, c2);
}

// floats in the order of unsigned numbers, zeros of either sign alike
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
constexpr uint32_t kOrderNegInf = 0x007FFFFFu;  // order_of(-inf)

// `publish`: what the thread has written is seen by who waits
template <bool publish>
__device__ __forceinline__ void cluster_arrive() {
  if (publish) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  else asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// The differences z - max are taken before the scaling by log2(e) / temperature: with rows masked by the type's lowest value, or far
// from zero, the product alone would overflow or lose the difference.
// A batch has a sum of its own, which is added to those before it with what the addition rounds off kept in `low`: a thread has up to 64
// batches, and equal terms round the same way (one running sum over rows of 2^22 words was off by up to 470 half steps of fp32).
template <class T, int NV>
__device__ __forceinline__ void add_batch(const uint4 (&raw)[NV], float c2, MaxSum& acc, float& low) {
  float m = acc.max;
#pragma unroll
  for (int j = 0; j < NV; ++j) m = fmaxf(m, vec_max<T>(raw[j]));
  const float ref = finite_ref(m);
  const float2 less = make_float2(-ref, -ref), by = make_float2(c2, c2);
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float f[kPerVec<T>];
    widen<T>(raw[j], f);
#pragma unroll
    for (int e = 0; e < kPerVec<T>; e += 2) {
      const float2 x = __fmul2_rn(__fadd2_rn(make_float2(f[e], f[e + 1]), less), by);
      sum = __fadd2_rn(sum, make_float2(exp2_fast(x.x), exp2_fast(x.y)));
    }
  }
  const float moved = exp2_fast((acc.max - ref) * c2), before = acc.sum * moved, batch = sum.x + sum.y;
  acc = {m, before + batch};
  low = low * moved + (before > batch ? batch - (acc.sum - before) : before - (acc.sum - batch));
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
// SCALED does not change when all of a row's log-probabilities move by one number, so its p are taken relative to the largest of them:
// a list of any mass, however far below (or above) what a number holds, then has P from 1 to k.

struct Part {  // a block's share of a row
  MaxSum rest, said;        // unlisted and listed words
  double mass, ent, cross;  // listed words: the sums of p, p ln p and p (z - said.max)
};
struct Whole {  // what the row's gradient needs; kept for it between loss and gradient
  float ref, a;         // unlisted words: a exp((z - ref) it)
  float max, inv_sum;   // q = exp((z - max) it) inv_sum
  float b, c;           // listed words: b q - c p
};
static_assert(sizeof(Whole) <= 4 * CVLC_DISTILL_STATS, "a row's place in the buffer");

// The library's functions, for what lies far out, are calls: in line, at every use, they cost short rows a tenth of their time (2503 rows of 397 words,
// the loss, 14.3 us, so 12.6).
__device__ __noinline__ double exp_far(double x) { return x > -(double)CUDART_INF_F && x < 0.0 ? fmax(exp(x), 4.9e-324) : exp(x); }  // of a number it is above 0
__device__ __noinline__ double ln_far(double x) { return log(x); }
// e^x to 2^-36 relative, which is far below what the rounding of x to fp32 leaves of it: x = n ln 2 + r, and the Taylor series of e^r
// (|r| <= 0.35: 0.35^11 / 11! = 2^-42).
__device__ __forceinline__ double exp_of(double x) {
  if (!(fabs(x) < 600.0)) return exp_far(x);
  const double n = rint(x * 1.4426950408889634074), r = fma(n, -0.693147180559945309417, x);
  double y = 1.0 / 3628800.0;
  y = fma(y, r, 1.0 / 362880.0);
  y = fma(y, r, 1.0 / 40320.0);
  y = fma(y, r, 1.0 / 5040.0);
  y = fma(y, r, 1.0 / 720.0);
  y = fma(y, r, 1.0 / 120.0);
  y = fma(y, r, 1.0 / 24.0);
  y = fma(y, r, 1.0 / 6.0);
  y = fma(y, r, 0.5);
  y = fma(y, r, 1.0);
  y = fma(y, r, 1.0);
  return __hiloint2double(__double2hiint(y) + ((int)n << 20), __double2loint(y));  // |n| < 870: the exponent stays a normal one's
}

// ln x to 2^-36: the fp32 logarithm, corrected by what its exponential leaves of x
__device__ __forceinline__ double ln_of(double x) {
  if (!(x > 1e-30 && x < 1e30)) return ln_far(x);
  const float y = logf((float)x);
  const double r = fma(x, exp_of((double)-y), -1.0);
  return (double)y + r * (1.0 - 0.5 * r);
}

// what p (z - a) has to gain to be p (z - b), a at most b; a = -inf: it is -inf already, or there is no mass
__device__ __forceinline__ double moved(double mass, float a, float b) {
  return a == -CUDART_INF_F || a == b ? 0.0 : mass * ((double)a - (double)b);
}

struct Sums {  // a row's parts joined
  MaxSum rest, said, all;
  double mass, left;  // left: what the bucket holds
  bool empty;         // every word is masked: no distribution
};
// by a warp: a lane for each part
__device__ __forceinline__ Sums sums_of(const Part* parts, uint32_t blocks, uint32_t rest, float c2) {
  const uint32_t lane = threadIdx.x & 31;
  Sums s = {{-CUDART_INF_F, 0.f}, {-CUDART_INF_F, 0.f}, {}, 0.0, 0.0, false};
  if (lane < blocks) s.rest = parts[lane].rest, s.said = parts[lane].said, s.mass = parts[lane].mass;
  for (uint32_t o = 1; o < blocks; o *= 2) {
    const MaxSum rest_o = {__shfl_xor_sync(kFull, s.rest.max, o), __shfl_xor_sync(kFull, s.rest.sum, o)};
    const MaxSum said_o = {__shfl_xor_sync(kFull, s.said.max, o), __shfl_xor_sync(kFull, s.said.sum, o)};
    s.mass += __shfl_xor_sync(kFull, s.mass, o);
    s.rest = join(s.rest, rest_o, c2);
    s.said = join(s.said, said_o, c2);
  }
  s.all = join(s.rest, s.said, c2);
  s.empty = s.all.max == -CUDART_INF_F && s.all.sum == 0.f;
  // without a word that it could stand for there is no bucket
  const bool some = !(s.rest.max == -CUDART_INF_F && s.rest.sum == 0.f);
  s.left = rest == CVLC_REST_BUCKET && some && s.mass < 1.0 ? 1.0 - s.mass : 0.0;
  return s;
}
__device__ __forceinline__ Whole whole_row(const Sums& s, uint32_t rest, float c2) {
  if (s.empty) return {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  Whole w;
  w.max = s.all.max;
  w.inv_sum = __frcp_rn(s.all.sum);
  w.b = (float)(s.mass + s.left);
  w.c = 1.f;
  if (rest == CVLC_REST_SCALED) {
    w.b = s.mass > 0.0 ? 1.f : (float)s.mass;  // (a NaN stays one)
    w.c = s.mass > 0.0 ? __frcp_rn((float)s.mass) : (float)s.mass;
  }
  const bool some = !(s.rest.max == -CUDART_INF_F && s.rest.sum == 0.f);
  w.ref = some ? s.rest.max : 0.f;
  w.a = some ? w.b * (exp2_fast((s.rest.max - s.all.max) * c2) * w.inv_sum) - (float)s.left * __frcp_rn(s.rest.sum) : 0.f;
  return w;
}
// by one thread
__device__ double loss_of(const Sums& s, const Part* parts, uint32_t blocks, uint32_t rest, float temperature) {
  if (s.empty) return 0.0;
  double ent = 0.0, cross = 0.0;
  for (uint32_t r = 0; r < blocks; ++r) {
    ent += parts[r].ent;
    cross += parts[r].cross + moved(parts[r].mass, parts[r].said.max, s.all.max);
  }
  const double it = 1.0 / (double)temperature, ln_sum = ln_of((double)s.all.sum);
  double loss = ent - cross * it + s.mass * ln_sum;
  if (rest == CVLC_REST_SCALED) loss = s.mass > 0.0 ? loss / s.mass - ln_of(s.mass) : s.mass;
  if (s.left > 0.0) loss += s.left * (ln_of(s.left) - (((double)s.rest.max - (double)s.all.max) * it + ln_of((double)s.rest.sum) - ln_sum));
  return loss;
}

// Records in shared memory: doubles first, then the places of the row's words, padded with -2 to whole sixteens.
__device__ __host__ __forceinline__ uint32_t padded(uint32_t k) { return (k + 15) & ~15u; }
__device__ __host__ __forceinline__ size_t records_bytes(uint32_t k) { return (size_t)padded(k) * (8 + 4 * 4); }
// What record i says of its word, where a word may have several: the sum over its records (`alone`: what each says by itself) in their
// order, by the first of them; below 0 for the others, which read nothing but their own (the first may already have put the sum
// in its place).  ln_p: its logarithm, `ln_alone` where the word has no other record.
__device__ __forceinline__ double said_by(const int* at, const double* alone, double ln_alone, uint32_t k, uint32_t i, double* ln_p) {
  const int here = at[i];
  double p = alone[i];
  bool merged = false, first = true;
  for (uint32_t o = 0; o < k && first; o += 16) {
    const int4* const q = reinterpret_cast<const int4*>(at + o);
    uint32_t same = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int4 v = q[j];
      same |= (v.x == here ? 1u : 0u) << (4 * j) | (v.y == here ? 2u : 0u) << (4 * j) | (v.z == here ? 4u : 0u) << (4 * j) |
              (v.w == here ? 8u : 0u) << (4 * j);
    }
    if (i >= o && i < o + 16) same &= ~(1u << (i - o));
    for (; same && first; same &= same - 1) {  // the lowest first
      const uint32_t other = o + __ffs(same) - 1;
      first = other > i;
      if (first) p += alone[other], merged = true;
    }
  }
  *ln_p = merged && first ? ln_of(p) : ln_alone;
  return first ? p : -1.0;
}
// what all of a row's log-probabilities are taken relative to, their largest being `top`
__device__ __forceinline__ double said_from(uint32_t rest, float top) { return rest == CVLC_REST_SCALED && top > -CUDART_INF_F ? (double)top : 0.0; }

// ---- a row's records, as a block sees them ----
// The words' places are marked as soon as the records are there, for the pass over the logits; what the teacher says of them is summed
// while the logits are on their way, and what the student says of them when they have come.
struct Records {
  int* at;        // places of the records in the block's share, or -1
  float* prob;    // their probabilities; below 0: counted with an earlier record of the word
  float* logit;   // the student's logits of their words
  float* said;    // the records' log-probabilities
  double* alone;  // their exponentials; then, for the first record of a word, the word's probability
  double mass, ent;

  __device__ __forceinline__ Records(unsigned char* shared, uint32_t k)
      : alone(reinterpret_cast<double*>(shared)), mass(0.0), ent(0.0) {
    at = reinterpret_cast<int*>(alone + padded(k));
    prob = reinterpret_cast<float*>(at + padded(k)), logit = prob + padded(k), said = logit + padded(k);
  }
  // the first record of a thread, and its word's logit
  int id;
  float logp, z;

  __device__ __forceinline__ void fetch(const DistillArgs& a, uint64_t row) {
    id = -1;
    logp = 0.f;
    if (threadIdx.x < a.k) {
      id = a.ids[row * a.k + threadIdx.x];
      logp = a.logp[row * a.k + threadIdx.x];
    }
  }
  // true: a word of this thread is marked twice.  marks: cleared before, a barrier between.  top_of_warp: the largest log-probability that
  // the warp has seen of all the row's words, whichever block has them
  template <class T>
  __device__ __forceinline__ bool mark(const DistillArgs& a, uint64_t row, const Row<T>& R, uint32_t* marks, float* top_of_warp) {
    bool twice = false;
    float top = -CUDART_INF_F;
    for (uint32_t i = threadIdx.x; i < a.k; i += blockDim.x) {
      if (i != threadIdx.x) id = a.ids[row * a.k + i], logp = a.logp[row * a.k + i];
      int p = -1;
      float v = 0.f;
      if (id >= 0 && (uint32_t)id >= a.vocab) {
        if (a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
      } else if (id >= 0) {
        top = fmaxf(top, logp);
        if ((p = R.place((uint32_t)id)) >= 0) {
          v = to_float(R.at[id]);
          const uint32_t bit = 1u << (p & 31);
          twice |= (atomicOr(marks + (p >> 5), bit) & bit) != 0;
        }
      }
      at[i] = p;
      said[i] = logp;
      if (i == threadIdx.x) z = v;
      else logit[i] = v;
    }
    if (threadIdx.x < padded(a.k) - a.k) at[a.k + threadIdx.x] = -2;
    if (a.rest == CVLC_REST_SCALED) {
      top = warp_max(top);
      if ((threadIdx.x & 31) == 0) top_of_warp[threadIdx.x >> 5] = top;
    }
    return twice;
  }
  // p of every word, summed in the order of its records; behind the barrier that follows mark()
  template <bool SUMS>
  __device__ __forceinline__ void teacher(const DistillArgs& a, bool twice, const float* top_of_warp) {
    float top = -CUDART_INF_F;
    if (a.rest == CVLC_REST_SCALED)
      for (uint32_t w = 0; w < blockDim.x / 32; ++w) top = fmaxf(top, top_of_warp[w]);
    const double from = said_from(a.rest, top);
    if (twice) {
      for (uint32_t i = threadIdx.x; i < a.k; i += blockDim.x) alone[i] = exp_of((double)said[i] - from);
      __syncthreads();
    }
    for (uint32_t i = threadIdx.x; i < a.k; i += blockDim.x) {
      double p = -1.0, ln_p = (double)said[i] - from;
      if (at[i] >= 0) {
        if (twice) p = said_by(at, alone, ln_p, a.k, i, &ln_p);
        else p = exp_of(ln_p);
        if (SUMS && !(p < 0.0)) {
          alone[i] = p;
          mass += p;
          if (p != 0.0) ent += p * ln_p;
        }
      }
      prob[i] = (float)p;  // (only this thread reads its own)
    }
  }
  // the sums of the warp's records; every lane has them
  __device__ __forceinline__ Part student(const DistillArgs& a, float c2) {
    if (threadIdx.x < a.k) logit[threadIdx.x] = z;
    Part p = {{}, {-CUDART_INF_F, 0.f}, 0.0, 0.0, 0.0};
    for (uint32_t i = threadIdx.x; i < a.k; i += blockDim.x)
      if (at[i] >= 0 && !(prob[i] < 0.f)) p.said.max = fmaxf(p.said.max, logit[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) p.said.max = fmaxf(p.said.max, __shfl_xor_sync(kFull, p.said.max, o));
    const float ref = finite_ref(p.said.max);
    for (uint32_t i = threadIdx.x; i < a.k; i += blockDim.x)
      if (at[i] >= 0 && !(prob[i] < 0.f)) {
        p.said.sum += exp2_fast((logit[i] - ref) * c2);
        if (alone[i] != 0.0) p.cross += alone[i] * ((double)logit[i] - (double)ref);  // (the logit may be far enough for any p above 0)
      }
    p.said.sum = warp_sum(p.said.sum), p.cross = warp_sum(p.cross), p.mass = warp_sum(mass), p.ent = warp_sum(ent);
    return p;
  }
};
__device__ __forceinline__ void add_said(Part& p, const Part& o, float c2) {
  const MaxSum all = join(p.said, o.said, c2);
  p.cross = p.cross + moved(p.mass, p.said.max, all.max) + o.cross + moved(o.mass, o.said.max, all.max);
  p.said = all;
  p.mass += o.mass, p.ent += o.ent;
}

// bits of the listed words of the block's vector i
template <class T>
__device__ __forceinline__ uint32_t listed_of(const uint8_t* marks, uint32_t i) {
  return kPerVec<T> == 8 ? marks[i] : (marks[i >> 1] >> ((i & 1) * 4)) & 15u;
}

// Latency bounds it: 16 rows of 32,000 words 10 us a call, 64 of 131,072 17.
// The loss goes through its share a batch ahead (2 x NV vectors of a thread in registers); the step keeps its batch for the gradient, and
// reads again what lies behind the first batch, if the row is longer than its cluster keeps.
template <class T, int NV, DistillKind KIND>
__global__ void __launch_bounds__(kRowThreads, 2) k_distill(DistillArgs a, uint32_t log_blocks, uint32_t mark_bytes) {
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ Part parts[kMaxClusterBlocks];
  __shared__ MaxSum of_warp[kRowThreads / 32];
  __shared__ Part said_of_warp[kRowThreads / 32];
  __shared__ float top_of_warp[kRowThreads / 32];
  __shared__ Whole whole;
  const uint32_t nt = blockDim.x, tid = threadIdx.x, blocks = 1u << log_blocks, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = blockIdx.x & (blocks - 1);
  const uint64_t row = blockIdx.x >> log_blocks;
  const Row<T> R(a.logits, row, a.row_stride, a.vocab, log_blocks, rank);
  const float weight = a.row_weight ? a.row_weight[row] : 1.f;
  const float c2 = a.c2;
  const uint32_t rounds = R.rounds();

  uint8_t* const marks = dyn;
  Records S(dyn + mark_bytes, a.k);

  // a row that counts for nothing is not looked at (but for what a later gradient may ask for)
  const bool idle = weight == 0.f && !(KIND == kDistillLoss && a.stats);

  uint4 raw[NV];
  if (!idle) {
    S.fetch(a, row);
    load_batch<T, NV>(R, 0, raw);
  }
  if (KIND != kDistillGrad && blocks > 1) cluster_arrive<false>();  // waited for before another block's shared memory is written
  if (!idle) {
    for (uint32_t i = tid; i < mark_bytes / 16; i += nt) reinterpret_cast<uint4*>(marks)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const bool twice = __syncthreads_or(S.mark<T>(a, row, R, reinterpret_cast<uint32_t*>(marks), top_of_warp));
    S.teacher<KIND != kDistillGrad>(a, twice, top_of_warp);
    if (KIND == kDistillGrad) {
      if (tid < a.k) S.logit[tid] = S.z;
    } else {
      MaxSum mine = {-CUDART_INF_F, 0.f};
      float low = 0.f;
      for (uint32_t from = 0;;) {
        uint4 ahead[NV];
        if (KIND == kDistillLoss && from + NV < rounds) load_batch<T, NV>(R, from + NV, ahead);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (from + j < rounds)
            if (const uint32_t bits = listed_of<T>(marks, tid + (from + j) * nt)) drop_elements<T>(raw[j], bits);
        add_batch<T, NV>(raw, c2, mine, low);
        from += NV;
        if (from >= rounds) break;
        if (KIND == kDistillLoss) {
#pragma unroll
          for (int j = 0; j < NV; ++j) raw[j] = ahead[j];
        } else {
          load_batch<T, NV>(R, from, raw);
        }
      }
      mine.sum += low;
      mine = warp_join(mine, c2);
      if (lane == 0) of_warp[warp] = mine;
      if (warp * 32 < a.k) {
        const Part p = S.student(a, c2);
        if (lane == 0) said_of_warp[warp] = p;
      }
      __syncthreads();
      if (warp == 0) {
        Part p = {{}, {-CUDART_INF_F, 0.f}, 0.0, 0.0, 0.0};
        const uint32_t with = min(nt / 32, (a.k + 31) / 32);  // warps that have records
        for (uint32_t w = 0; w < with; ++w) add_said(p, said_of_warp[w], c2);
        p.rest = join_warps(of_warp, nt / 32, c2);
        if (blocks == 1) {
          if (lane == 0) parts[0] = p;
        } else {
          cluster_wait();
          if (lane < blocks) *cg::this_cluster().map_shared_rank(&parts[rank], lane) = p;
          cluster_arrive<true>();
        }
      } else if (blocks > 1) {
        cluster_wait();
        cluster_arrive<false>();
      }
    }
  } else if (KIND != kDistillGrad && blocks > 1) {
    cluster_wait();
    cluster_arrive<false>();
  }
  if (KIND != kDistillGrad) {
    if (blocks > 1) cluster_wait();
    else __syncthreads();
  }
  Whole w = {};
  if (KIND == kDistillGrad) {
    if (!idle) w = *reinterpret_cast<const Whole*>(a.stats + row * CVLC_DISTILL_STATS);
  } else if (KIND == kDistillLoss) {
    if (warp != 0 || rank != 0) return;
    double loss = 0.0;
    if (!idle) {
      const Sums s = sums_of(parts, blocks, a.rest, c2);
      if (lane == 0) loss = loss_of(s, parts, blocks, a.rest, a.temperature);
      if (lane == 0 && a.stats) *reinterpret_cast<Whole*>(a.stats + row * CVLC_DISTILL_STATS) = whole_row(s, a.rest, c2);
    }
    if (lane == 0) a.loss[row] = weight == 0.f ? 0.f : (float)((double)weight * loss);
    return;
  } else if (!idle) {
    if (warp == 0) {
      const Whole mine = whole_row(sums_of(parts, blocks, a.rest, c2), a.rest, c2);
      if (lane == 0) whole = mine;
    }
    __syncthreads();
    w = whole;
  }

  // the gradient, a vector at a time; where logits and gradient lie differently against 16 bytes, by elements
  T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
  const bool alike = ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(R.at)) & 15) == 0;
  const float scale = idle ? 0.f : weight / a.temperature;
  const float ca = w.a * scale;
  for (uint32_t from = 0; from < rounds; from += NV) {
    if (!idle && (KIND == kDistillGrad ? from > 0 : rounds > NV)) load_batch<T, NV>(R, from, raw);
    const uint32_t v0 = R.first + from * R.apart;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float f[kPerVec<T>];
      widen<T>(raw[j], f);
#pragma unroll
      for (int e = 0; e < kPerVec<T>; e += 2) {
        const float2 x = __fmul2_rn(__fadd2_rn(make_float2(f[e], f[e + 1]), make_float2(-w.ref, -w.ref)), make_float2(c2, c2));
        const float2 y = __fmul2_rn(make_float2(exp2_fast(x.x), exp2_fast(x.y)), make_float2(ca, ca));
        f[e] = y.x, f[e + 1] = y.y;
      }
      raw[j] = idle ? make_uint4(0, 0, 0, 0) : narrow<T>(f);
    }
    uint4* const to = reinterpret_cast<uint4*>(g - R.lead);
    if (alike) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (R.whole(v0 + j * R.apart)) __stcs(to + v0 + j * R.apart, raw[j]);
    }
    if (!alike || R.ragged()) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const uint32_t v = v0 + j * R.apart;
        if (v >= R.vecs || (alike && R.whole(v))) continue;
        const int word = R.word(v);
        const T* const elements = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
        for (int e = 0; e < kPerVec<T>; ++e)
          if (word + e >= 0 && word + e < (int)R.vocab) g[word + e] = elements[e];
      }
    }
  }
  if (!idle) {
    __syncthreads();  // the listed words' gradients replace what the vectors hold in their places
    const float cb = w.b * scale, cc = w.c * scale;
    for (uint32_t i = tid; i < a.k; i += nt)
      if (S.at[i] >= 0 && !(S.prob[i] < 0.f)) {
        const float q = exp2_fast((S.logit[i] - w.max) * c2) * w.inv_sum;
        g[a.ids[row * a.k + i]] = from_float<T>(cb * q - cc * S.prob[i]);
      }
  }
  // the loss last: its logarithms take as long as a store
  if (KIND == kDistillStep && rank == 0 && warp == 0) {
    double loss = 0.0;
    if (!idle) {
      const Sums s = sums_of(parts, blocks, a.rest, c2);
      if (lane == 0) loss = loss_of(s, parts, blocks, a.rest, a.temperature);
    }
    if (lane == 0) a.loss[row] = weight == 0.f ? 0.f : (float)((double)weight * loss);
  }
}

// ---- many long rows: a block goes from row to row ----
//
// Everything that a row needs beside its elements (records, sums, logarithms) takes a block about as long as reading 64 KB does, whoever does
// it.  So where rows are many it is done by warps of their own, beside the pass over the elements: a row's records are prepared while
// the row before it is passed over, and its loss, its listed words and its ragged ends are finished while the row behind it is.  One
// thread copies the rows through a ring of stages in shared memory (cp.async.bulk), four vectors of every thread a stage.  The step passes over
// every row twice, at first over what the ring still holds of it, then over what it has to copy once more, most of which is in the L2 cache
// (the 296 rows on their way are 76 MB at 131,072 words of 16 bits).  Keeping the row in the cluster's registers instead costs every block of the cluster all of the above:
// 4096 x 131072 bf16 750 us, so 430 to 455 (of 332 at the copy bandwidth; from box to box); the loss 200 to 215 (of 166).  The pass is a
// chain of load, maximum, exponential and sum in 16 warps an SM: without the exponentials the loss takes 156 us.  More warps for it leave
// too few registers and stages (ten 211, twelve 243).
constexpr int kStreamWarps = 8, kSideWarps = 4;  // and one that copies
constexpr int kStreamLanes = kStreamWarps * 32, kSideLanes = kSideWarps * 32;
constexpr int kStreamBlock = kStreamLanes + kSideLanes + 32;
constexpr int kPrepWarps = kSideWarps - 1, kPrepLanes = kPrepWarps * 32;  // distillation: the side warp that is left has the losses
constexpr int kRecordsAhead = 4;  // records of a side thread whose loads are on their way
constexpr int kStageShare = 4;  // vectors of a thread in a stage: with two, waiting for it and giving it back were a third of the instructions
constexpr int kStageVecs = kStageShare * kStreamLanes;  // 16 KB
constexpr int kStagesMost = 8;
constexpr size_t kStreamShared = 110 * 1024;  // of a block, two of which share an SM

struct RowAt {  // where a row lies
  const unsigned char* from;  // vector 0
  uint32_t lead, vecs, whole_from, wholes;
};
template <class T>
__device__ __forceinline__ RowAt row_at(const DistillArgs& a, uint64_t row) {
  const T* const at = static_cast<const T*>(a.logits) + row * a.row_stride;
  RowAt r;
  r.lead = (uint32_t)((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(T));
  r.from = reinterpret_cast<const unsigned char*>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)15);
  r.vecs = (r.lead + a.vocab + kPerVec<T> - 1) / kPerVec<T>;
  r.whole_from = r.lead ? 1 : 0;
  const uint32_t whole_to = (r.lead + a.vocab) / kPerVec<T>;
  r.wholes = whole_to > r.whole_from ? whole_to - r.whole_from : 0;
  return r;
}

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(shared_at(b)), "r"(n)); }
__device__ __forceinline__ void bar_arrive(uint64_t* b) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(shared_at(b)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(shared_at(b)), "r"(bytes) : "memory");
}
// The side warps and the copying one come first: the scheduler prefers older warps, and those of the pass over the elements always have something
// to do (with them first, the side warps took 20 us for 2 us of work, and the rows waited).
constexpr int kStreamFirst = kSideLanes + 32;
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile("{.reg .pred p;\n mbarrier.try_wait.parity.shared.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;}"
               : "=r"(done)
               : "r"(shared_at(b)), "r"(parity)
               : "memory");
  return done != 0;
}
__device__ __forceinline__ uint64_t nanoseconds() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// What a block's waits share.  They are bounded.  When one has run out, the copying thread stops, by its own wait or because it is told, and
// who has waited for a copy goes on only then, without waiting any more: so a stage that may still be read is never written, whoever
// gives it back.  The rows that are not finished are void.
constexpr uint64_t kWaitMost = 4000000000ull;  // nanoseconds
constexpr int kLateTries = 256;                // behind that: the time also runs while the block does not (another process has the GPU)
struct Waits {
  uint32_t *gone, *stopped;  // in shared memory, 0 at first: a wait has run out; nothing will be copied any more
  int32_t* status;           // or nullptr
  uint64_t most;
  __device__ __forceinline__ bool over() const { return *static_cast<volatile uint32_t*>(gone) != 0; }
  __device__ __forceinline__ void stop() const { *static_cast<volatile uint32_t*>(stopped) = 1; }
};
// The time is over; false: the wait has run out
__device__ __forceinline__ bool wait_late(uint64_t* b, uint32_t parity, Waits w, bool copies) {
  for (int i = 0; i < kLateTries; ++i)
    if (bar_try(b, parity)) return true;
  *static_cast<volatile uint32_t*>(w.gone) = 1;
  if (w.status) set_status(w.status, CVLC_ERR_DEVICE_TIMEOUT);
  const uint64_t began = nanoseconds();
  while (!copies && !*static_cast<volatile uint32_t*>(w.stopped) && nanoseconds() - began < 2 * w.most) {
  }
  return false;
}
// Clears `ok` when it runs out; later ones try once.
__device__ __forceinline__ void bar_wait(uint64_t* b, uint32_t parity, const Waits& w, bool& ok) {
  if (bar_try(b, parity)) return;
  const uint64_t began = nanoseconds();
  while (ok) {
    if (bar_try(b, parity)) return;
    if (nanoseconds() - began > w.most) {
      ok = wait_late(b, parity, w, false);
      return;
    }
  }
}
// ... of the copying thread, which also stops when another's has
__device__ __forceinline__ bool copy_wait(uint64_t* b, uint32_t parity, const Waits& w) {
  if (bar_try(b, parity)) return true;
  const uint64_t began = nanoseconds();
  while (!w.over()) {
    if (bar_try(b, parity)) return true;
    if (nanoseconds() - began > w.most) return wait_late(b, parity, w, true);
  }
  return false;
}
// A warp has read its part of a stage.  The copy that fills the stage next writes it by another path than the loads take: the loads
// have to be over before the copying thread hears of it, and the arrival alone does not see to that.
__device__ __forceinline__ void release_stage(uint64_t* b) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if ((threadIdx.x & 31) == 0) bar_arrive(b);
}
// named barriers among some of a block's warps
template <int N>
__device__ __forceinline__ void some_sync(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(N) : "memory"); }
template <int N>
__device__ __forceinline__ void some_arrive(int id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(N) : "memory"); }
template <int N>
__device__ __forceinline__ bool some_or(int id, bool v) {
  uint32_t r;
  asm volatile("{.reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, %3, p;\n selp.u32 %0, 1, 0, q;}" : "=r"(r) : "r"((uint32_t)v), "r"(id), "n"(N) : "memory");
  return r != 0;
}
template <int N>
__device__ __forceinline__ uint32_t some_count(int id, bool v) {
  uint32_t r;
  asm volatile("{.reg .pred p;\n setp.ne.u32 p, %1, 0;\n bar.red.popc.u32 %0, %2, %3, p;}" : "=r"(r) : "r"((uint32_t)v), "r"(id), "n"(N) : "memory");
  return r;
}
enum { kBarSide = 1, kBarStream = 2, kBarReady = 3, kBarDone = 5, kBarLoss = 7 };  // from kBarReady on: one for each of two rows

// of a row's whole vectors, those that the ring no longer holds when it has passed
__device__ __forceinline__ uint32_t copied_again(uint32_t wholes, uint32_t stages) {
  const uint32_t cuts = (wholes + kStageVecs - 1) / kStageVecs;
  return cuts > stages ? (cuts - stages) * kStageVecs : 0;
}
// The copying thread: the whole vectors of the block's rows through the ring; with two passes all but what the ring still holds of the row a
// second time.  The last reading of a row leaves nothing in the L2 cache.
template <class T, int PASSES, class F>
__device__ void copy_rows(const DistillArgs& a, uint64_t rows, uint4* ring, uint32_t stages, uint64_t* full, uint64_t* empty, const Waits& waits, F&& skip) {
  uint64_t once;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
  uint32_t stage = 0, phase = 0;
  bool ok = true, skip_next = skip(blockIdx.x);
  for (uint64_t row = blockIdx.x; ok && row < rows; row += gridDim.x) {
    const bool skipped = skip_next;
    skip_next = skip(row + gridDim.x);  // known before it is needed
    if (skipped) continue;
    const RowAt R = row_at<T>(a, row);
    for (int pass = 0; ok && pass < PASSES; ++pass) {
      const uint32_t to_copy = pass == 0 ? R.wholes : copied_again(R.wholes, stages);
      const bool once_more = pass + 1 < PASSES;
      for (uint32_t v = 0; v < to_copy; v += kStageVecs) {
        ok = copy_wait(&empty[stage], phase ^ 1, waits);
        if (!ok) break;
        const uint32_t bytes = min(R.wholes - v, (uint32_t)kStageVecs) * 16;
        bar_expect(&full[stage], bytes);
        const unsigned char* const src = R.from + ((size_t)R.whole_from + v) * 16;
        const uint32_t to = shared_at(ring + (size_t)stage * kStageVecs), bar = shared_at(&full[stage]);
        if (!once_more || v >= copied_again(R.wholes, stages))
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(to), "l"(src),
                       "r"(bytes), "r"(bar), "l"(once)
                       : "memory");
        else
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(src), "r"(bytes), "r"(bar)
                       : "memory");
        if (++stage == stages) stage = 0, phase ^= 1;
      }
    }
  }
  // no copy is left on its way: all stages have been given back, or, where a wait has run out, have been filled
  const uint32_t next = stage, next_phase = phase;
  for (uint32_t i = 0; ok && i < stages; ++i) {
    ok = copy_wait(&empty[stage], phase ^ 1, waits);
    if (++stage == stages) stage = 0, phase ^= 1;
  }
  if (ok) return;
  waits.stop();
  uint32_t alone = 0;
  stage = next, phase = next_phase;
  for (uint32_t i = 0; i < stages; ++i) {  // (of a stage that has never been filled the phase before the first is complete)
    (void)copy_wait(&full[stage], phase ^ 1, Waits{&alone, nullptr, nullptr, waits.most});
    if (++stage == stages) stage = 0, phase ^= 1;
  }
}
// word of a row's i-th element beside its whole vectors (E of the first vector, then E of the last one), or -1
template <int E>
__device__ __forceinline__ int end_word(const RowAt& R, uint32_t vocab, uint32_t i) {
  const uint32_t last = R.vecs - 1;
  if (i >= 2 * E || !(i < E ? R.whole_from > 0 || R.wholes == 0 : last > 0 && last >= R.whole_from + R.wholes)) return -1;
  const int w = i < E ? (int)i - (int)R.lead : (int)(last * E + i - E) - (int)R.lead;
  return w >= 0 && w < (int)vocab ? w : -1;
}

// The warp's part of a stage that holds the row's whole vectors from `v` on; what lies behind them is minus infinity.
template <class T>
__device__ __forceinline__ void read_stage(const uint4* ring, uint32_t stage, uint32_t v, uint32_t wholes, uint4 (&raw)[kStageShare]) {
  const uint32_t tid = threadIdx.x - kStreamFirst;
  const uint4* const from = ring + stage * kStageVecs + tid;
  if (v + kStageVecs <= wholes) {
#pragma unroll
    for (int j = 0; j < kStageShare; ++j) raw[j] = from[j * kStreamLanes];
  } else {
#pragma unroll
    for (int j = 0; j < kStageShare; ++j) {
      raw[j] = nothing<T>();
      if (v + tid + j * kStreamLanes < wholes) raw[j] = from[j * kStreamLanes];
    }
  }
}
// ... of the next stage of the ring, which is then given back, unless it is to be read once more
template <class T>
__device__ __forceinline__ void take_stage(const uint4* ring, uint32_t& stage, uint32_t& phase, uint32_t stages, uint64_t* full, uint64_t* empty,
                                           uint32_t v, uint32_t wholes, const Waits& waits, bool& ok, uint4 (&raw)[kStageShare], bool keep = false) {
  bar_wait(&full[stage], phase, waits, ok);
  read_stage<T>(ring, stage, v, wholes, raw);
  if (!keep) release_stage(&empty[stage]);
  if (++stage == stages) stage = 0, phase ^= 1;
}
// add_batch() of vectors whose largest element is known; the sum moves only when the maximum does
template <class T>
__device__ __forceinline__ void add_share(const uint4 (&raw)[kStageShare], float largest, float c2, MaxSum& acc) {
  if (largest > acc.max) {
    acc.sum *= exp2_fast((acc.max - largest) * c2);
    acc.max = largest;
  }
  const float ref = finite_ref(acc.max);
  const float2 less = make_float2(-ref, -ref), by = make_float2(c2, c2);
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < kStageShare; ++j) {
    float f[kPerVec<T>];
    widen<T>(raw[j], f);
#pragma unroll
    for (int e = 0; e < kPerVec<T>; e += 2) {
      const float2 x = __fmul2_rn(__fadd2_rn(make_float2(f[e], f[e + 1]), less), by);
      sum = __fadd2_rn(sum, make_float2(exp2_fast(x.x), exp2_fast(x.y)));
    }
  }
  acc.sum += sum.x + sum.y;
}

struct RowSide {  // what the side warps know of a row
  MaxSum said, ends;        // listed words; unlisted ones in the ragged ends
  double mass, ent, cross;  // as in Part
  float left, b_left, b, c; // left of the bucket, if there is one; b with and without it; c
  MaxSum rest[kStreamWarps];
};

// The row's numbers, by a whole warp
__device__ __forceinline__ Whole whole_of(const RowSide& s, float c2, MaxSum* rest_out, MaxSum* all_out, float* left_out) {
  const uint32_t lane = threadIdx.x & 31;
  const MaxSum mine = lane < kStreamWarps ? s.rest[lane] : lane == kStreamWarps ? s.ends : MaxSum{-CUDART_INF_F, 0.f};
  const MaxSum rest = warp_join(mine, c2);
  const MaxSum all = join(rest, s.said, c2);
  const bool some = !(rest.max == -CUDART_INF_F && rest.sum == 0.f);  // without a word that it could stand for there is no bucket
  const float left = some ? s.left : 0.f;
  *rest_out = rest, *all_out = all, *left_out = left;
  if (all.max == -CUDART_INF_F && all.sum == 0.f) return {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};  // every word is masked
  Whole w;
  w.max = all.max;
  w.inv_sum = __frcp_rn(all.sum);
  w.b = some ? s.b_left : s.b;
  w.c = s.c;
  w.ref = some ? rest.max : 0.f;
  w.a = some ? w.b * (exp2_fast((rest.max - all.max) * c2) * w.inv_sum) - left * __frcp_rn(rest.sum) : 0.f;
  return w;
}

// thread `t` of `nt` writes its part of a row of zeros
template <class T>
__device__ __forceinline__ void zero_row(T* g, uint32_t vocab, uint32_t t, uint32_t nt) {
  const uint32_t lead = (uint32_t)(-(reinterpret_cast<uintptr_t>(g) / sizeof(T)) & (kPerVec<T> - 1)), front = min(lead, vocab);
  const uint32_t vecs = (vocab - front) / kPerVec<T>, back = front + vecs * kPerVec<T>;
  if (t < front) g[t] = from_float<T>(0.f);
  for (uint32_t v = t; v < vecs; v += nt) __stcs(reinterpret_cast<uint4*>(g + front) + v, make_uint4(0, 0, 0, 0));
  if (back + t < vocab) g[back + t] = from_float<T>(0.f);
}

template <class T, DistillKind KIND>
__global__ void __launch_bounds__(kStreamBlock, 2) k_distill_stream(DistillArgs a, uint32_t stages, uint32_t mark_bytes) {
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ uint64_t full[kStagesMost], empty[kStagesMost];
  __shared__ RowSide sides[2];
  __shared__ Part of_side[kPrepWarps];
  __shared__ float top_of_side[kPrepWarps];
  __shared__ uint32_t gone, stopped;
  constexpr int E = kPerVec<T>;
  const uint32_t thread = threadIdx.x, lane = thread & 31;
  const float c2 = a.c2;
  uint4* const ring = reinterpret_cast<uint4*>(dyn);
  const auto marks_of = [&](uint32_t buf) { return dyn + stages * (kStageVecs * 16) + buf * mark_bytes; };
  const auto records_of = [&](uint32_t buf) {  // of two rows, as in Records
    return reinterpret_cast<double*>(dyn + stages * (kStageVecs * 16) + 2 * mark_bytes + buf * (uint32_t)records_bytes(a.k));
  };
  const auto weight_of = [&](uint64_t row) { return !a.row_weight ? 1.f : row < a.rows ? a.row_weight[row] : 0.f; };
  const bool all_rows = KIND == kDistillLoss && a.stats;  // a later gradient may ask for rows that count for nothing
  const Waits waits = {&gone, &stopped, a.status, kWaitMost};

  if (thread == 0) {
    gone = stopped = 0;
    for (uint32_t i = 0; i < stages; ++i) bar_init(&full[i], 1), bar_init(&empty[i], kStreamWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (uint32_t i = thread; i < mark_bytes / 8; i += kStreamBlock) reinterpret_cast<uint4*>(marks_of(0))[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();

  bool ok = true;
  if (thread >= kSideLanes && thread < kStreamFirst) {
    if (lane == 0)
      copy_rows<T, KIND == kDistillStep ? 2 : 1>(a, a.rows, ring, stages, full, empty, waits, [&](uint64_t row) { return !all_rows && weight_of(row) == 0.f; });
    return;
  }

  if (thread < kSideLanes) {
    // ---- the side warps: records, ragged ends, losses ----
    const uint32_t t = thread, side = t >> 5;
    const auto end_of = [&](const RowAt& R) { return side == 0 ? end_word<E>(R, a.vocab, lane) : -1; };
    // A row's records begin with loads that depend on each other: the first record of a thread is fetched while an earlier row is worked on,
    // and its word's logit after it.
    struct First {
      int id, end;
      float logp, z, end_z;
    };
    const auto fetch = [&](uint64_t row, First& f) {
      f.id = -1, f.logp = 0.f;
      if (row < a.rows && t < a.k) f.id = a.ids[row * a.k + t], f.logp = a.logp[row * a.k + t];
    };
    const auto fetch_logits = [&](uint64_t row, First& f) {
      if (row >= a.rows) return;
      const RowAt R = row_at<T>(a, row);
      const T* const z = reinterpret_cast<const T*>(R.from) + R.lead;
      f.end = end_of(R);
      f.end_z = f.end >= 0 ? to_float(z[f.end]) : -CUDART_INF_F;
      f.z = f.id >= 0 && (uint32_t)f.id < a.vocab ? to_float(z[f.id]) : 0.f;
    };
    const auto prepare = [&](uint64_t row, uint32_t buf, const First& first, bool again) {
      some_sync<kPrepLanes>(kBarSide);  // the row before the last one is finished, its marks cleared
      const RowAt R = row_at<T>(a, row);
      const T* const z = reinterpret_cast<const T*>(R.from) + R.lead;
      uint8_t* const marks = marks_of(buf);
      double* const alone = records_of(buf);
      int* const at = reinterpret_cast<int*>(alone + padded(a.k));
      float* const prob = reinterpret_cast<float*>(at + padded(a.k));
      float* const logit = prob + padded(a.k);
      float* const said = logit + padded(a.k);
      bool twice = false;
      float top = -CUDART_INF_F;
      const int end = first.end;
      const float end_z = first.end_z;
      for (uint32_t base = t; base < a.k; base += kRecordsAhead * kPrepLanes) {  // a few records of a thread at once: their loads are far
        int ids[kRecordsAhead];
        float lps[kRecordsAhead], zs[kRecordsAhead];
#pragma unroll
        for (int j = 0; j < kRecordsAhead; ++j) {
          const uint32_t i = base + j * kPrepLanes;
          const bool fetched = i == t;
          ids[j] = fetched ? first.id : i < a.k ? a.ids[row * a.k + i] : -1;
          lps[j] = fetched ? first.logp : i < a.k ? a.logp[row * a.k + i] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kRecordsAhead; ++j)
          zs[j] = base + j * kPrepLanes == t ? first.z : ids[j] >= 0 && (uint32_t)ids[j] < a.vocab ? to_float(z[ids[j]]) : 0.f;
#pragma unroll
        for (int j = 0; j < kRecordsAhead; ++j) {
          const uint32_t i = base + j * kPrepLanes;
          if (i >= a.k) break;
          int p = -1;
          if (ids[j] >= 0 && (uint32_t)ids[j] >= a.vocab) {
            if (a.status) set_status(a.status, CVLC_ERR_INVALID_ARG);
          } else if (ids[j] >= 0) {
            p = ids[j] + (int)R.lead;
            top = fmaxf(top, lps[j]);
            const uint32_t bit = 1u << (p & 31);
            twice |= (atomicOr(reinterpret_cast<uint32_t*>(marks) + (p >> 5), bit) & bit) != 0;
          }
          at[i] = p, said[i] = lps[j], logit[i] = zs[j];
        }
      }
      if (t < padded(a.k) - a.k) at[a.k + t] = -2;
      if (a.rest == CVLC_REST_SCALED) {
        top = warp_max(top);
        if (lane == 0) top_of_side[side] = top;  // (the last row's were read before this row's first barrier)
      }
      twice = some_or<kPrepLanes>(kBarSide, twice);
      if (a.rest == CVLC_REST_SCALED)
        for (int w = 0; w < kPrepWarps; ++w) top = fmaxf(top, top_of_side[w]);
      const double from = said_from(a.rest, top);
      Part mine = {{-CUDART_INF_F, 0.f}, {-CUDART_INF_F, 0.f}, 0.0, 0.0, 0.0};
      if (twice) {
        for (uint32_t i = t; i < a.k; i += kPrepLanes) alone[i] = exp_of((double)said[i] - from);
        some_sync<kPrepLanes>(kBarSide);
      }
      for (uint32_t i = t; i < a.k; i += kPrepLanes) {
        double p = -1.0, ln_p = (double)said[i] - from;
        if (at[i] >= 0) {
          if (twice) p = said_by(at, alone, ln_p, a.k, i, &ln_p);
          else p = exp_of(ln_p);
          if (KIND != kDistillGrad && !(p < 0.0)) {
            alone[i] = p;
            mine.mass += p;
            if (p != 0.0) mine.ent += p * ln_p;
            mine.said.max = fmaxf(mine.said.max, logit[i]);
          }
        }
        prob[i] = (float)p;  // (only this thread reads its own)
      }
      if (KIND != kDistillGrad) {
#pragma unroll
        for (int o = 16; o; o >>= 1) mine.said.max = fmaxf(mine.said.max, __shfl_xor_sync(kFull, mine.said.max, o));
        const float ref = finite_ref(mine.said.max);
        for (uint32_t i = t; i < a.k; i += kPrepLanes)
          if (at[i] >= 0 && !(prob[i] < 0.f)) {
            mine.said.sum += exp2_fast((logit[i] - ref) * c2);
            if (alone[i] != 0.0) mine.cross += alone[i] * ((double)logit[i] - (double)ref);
          }
        mine.said.sum = warp_sum(mine.said.sum), mine.mass = warp_sum(mine.mass), mine.ent = warp_sum(mine.ent), mine.cross = warp_sum(mine.cross);
        if (side == 0) {
          const bool listed = end >= 0 && (marks[(end + R.lead) >> 3] >> ((end + R.lead) & 7) & 1);
          const float e = listed ? -CUDART_INF_F : end_z;
          mine.rest = warp_join(MaxSum{e, e == -CUDART_INF_F ? 0.f : e == e ? 1.f : e}, c2);
        }
        if (lane == 0) of_side[side] = mine;
        if (again) some_sync<kSideLanes>(kBarLoss + buf);  // the loss of the row before the last one is done
        some_sync<kPrepLanes>(kBarSide);
        if (t == 0) {
          Part p = of_side[0];
          for (int w = 1; w < kPrepWarps; ++w) add_said(p, of_side[w], c2);
          RowSide& s = sides[buf];
          s.said = p.said, s.ends = p.rest;
          s.mass = p.mass, s.ent = p.ent, s.cross = p.cross;
          const double left = a.rest == CVLC_REST_BUCKET && p.mass < 1.0 ? 1.0 - p.mass : 0.0;
          s.left = (float)left;
          s.b_left = (float)(p.mass + left), s.b = (float)p.mass, s.c = 1.f;
          if (a.rest == CVLC_REST_SCALED) {
            s.b = s.b_left = p.mass > 0.0 ? 1.f : (float)p.mass;  // (a NaN stays one)
            s.c = p.mass > 0.0 ? __frcp_rn((float)p.mass) : (float)p.mass;
          }
        }
      }
      __threadfence_block();
      some_arrive<kStreamLanes + kPrepLanes>(kBarReady + buf);
    };
    const auto finish = [&](uint64_t row, uint32_t buf) {
      some_sync<kStreamLanes + kSideLanes>(kBarDone + buf);
      const RowAt R = row_at<T>(a, row);
      const float weight = a.row_weight ? a.row_weight[row] : 1.f;
      uint8_t* const marks = marks_of(buf);
      int* const at = reinterpret_cast<int*>(records_of(buf) + padded(a.k));
      float* const prob = reinterpret_cast<float*>(at + padded(a.k));
      float* const logit = prob + padded(a.k);
      Whole w;
      if (KIND == kDistillGrad) {
        w = *reinterpret_cast<const Whole*>(a.stats + row * CVLC_DISTILL_STATS);
      } else {
        MaxSum rest, all;
        float left;
        if (KIND == kDistillStep) w = whole_of(sides[buf], c2, &rest, &all, &left);
      }
      T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
      const float scale = weight / a.temperature;
      if (KIND != kDistillLoss) {
        if (waits.over()) w.a = w.b = CUDART_NAN_F;
        const int end = end_of(R);
        if (end >= 0 && !(marks[(end + R.lead) >> 3] >> ((end + R.lead) & 7) & 1)) {
          const float z = to_float((reinterpret_cast<const T*>(R.from) + R.lead)[end]);
          g[end] = from_float<T>(w.a * scale * exp2_fast((z - w.ref) * c2));
        }
        for (uint32_t i = t; i < a.k; i += kPrepLanes)
          if (at[i] >= 0 && !(prob[i] < 0.f)) {
            const float q = exp2_fast((logit[i] - w.max) * c2) * w.inv_sum;
            g[at[i] - (int)R.lead] = from_float<T>(w.b * scale * q - w.c * scale * prob[i]);
          }
        some_sync<kPrepLanes>(kBarSide);  // the ends' marks have been read
      }
      for (uint32_t i = t; i < a.k; i += kPrepLanes)
        if (at[i] >= 0) reinterpret_cast<uint32_t*>(marks)[at[i] >> 5] = 0;
    };
    // the next row that counts, whose loss is 0 where it does not
    const auto counting = [&](uint64_t row) {
      for (; row < a.rows && !all_rows && weight_of(row) == 0.f; row += gridDim.x)
        if (KIND != kDistillGrad && t == 0) a.loss[row] = 0.f;
      return row;
    };
    if (side == kPrepWarps) {
      // ---- the losses: their logarithms in 64 bits take a lane as long as the records take the others ----
      if (KIND == kDistillGrad) {  // (it has none, but the barriers count it)
        uint32_t buf = 0;
        for (uint64_t row = counting(blockIdx.x); row < a.rows; row = counting(row + gridDim.x), buf ^= 1)
          some_sync<kStreamLanes + kSideLanes>(kBarDone + buf);
        return;
      }
      uint32_t buf = 0;
      for (uint64_t row = counting(blockIdx.x); row < a.rows; row = counting(row + gridDim.x), buf ^= 1) {
        const float weight = weight_of(row);
        some_sync<kStreamLanes + kSideLanes>(kBarDone + buf);
        const RowSide& s = sides[buf];
        MaxSum rest, all;
        float left;
        const Whole w = whole_of(s, c2, &rest, &all, &left);
        if (lane == 0) {
          double loss = 0.0;
          if (!(all.max == -CUDART_INF_F && all.sum == 0.f)) {
            const double it = 1.0 / (double)a.temperature, ln_sum = ln_of((double)all.sum);
            loss = s.ent - (s.cross + moved(s.mass, s.said.max, all.max)) * it + s.mass * ln_sum;
            if (a.rest == CVLC_REST_SCALED) loss = s.mass > 0.0 ? loss / s.mass - ln_of(s.mass) : s.mass;
            if (left > 0.f) {
              const double l = 1.0 - s.mass;
              loss += l * (ln_of(l) - (((double)rest.max - (double)all.max) * it + ln_of((double)rest.sum) - ln_sum));
            }
          }
          if (waits.over()) loss = CUDART_NAN;
          a.loss[row] = weight == 0.f ? 0.f : (float)((double)weight * loss);
          if (KIND == kDistillLoss && a.stats) *reinterpret_cast<Whole*>(a.stats + row * CVLC_DISTILL_STATS) = w;
        }
        __syncwarp();
        some_arrive<kSideLanes>(kBarLoss + buf);  // the row's sums have been read
      }
      return;
    }
    uint64_t before = ~0ull, row = counting(blockIdx.x);
    uint32_t buf = 0, prepared = 0;
    First first, next;
    fetch(row, first);
    fetch_logits(row, first);
    while (row < a.rows) {
      const uint64_t after = counting(row + gridDim.x);
      fetch(after, next);
      prepare(row, buf, first, prepared >= 2);
      ++prepared;
      fetch_logits(after, next);
      if (before != ~0ull) finish(before, buf ^ 1);
      before = row, row = after, first = next;
      buf ^= 1;
    }
    if (before != ~0ull) finish(before, buf ^ 1);
    if (KIND != kDistillGrad)
      for (uint32_t i = 0; i < min(prepared, 2u); ++i) some_sync<kSideLanes>(kBarLoss + ((prepared - 1 - i) & 1));  // no barrier is left half full
    return;
  }

  // ---- the pass over the elements ----
  const uint32_t tid = thread - kStreamFirst;
  uint32_t stage = 0, phase = 0, buf = 0;
  float next_weight = weight_of(blockIdx.x);
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float weight = next_weight;
    next_weight = weight_of(row + gridDim.x);
    const RowAt R = row_at<T>(a, row);
    T* const g = static_cast<T*>(a.grad) + row * a.grad_stride;
    if (!all_rows && weight == 0.f) {
      if (KIND != kDistillLoss) zero_row<T>(g, a.vocab, tid, kStreamLanes);
      continue;
    }
    some_sync<kStreamLanes + kPrepLanes>(kBarReady + buf);
    const unsigned char* const marks = marks_of(buf);
    const uint32_t again = copied_again(R.wholes, stages);  // from here on the ring still holds the row for the second pass
    Whole w = {};
    if (KIND != kDistillGrad) {
      MaxSum acc = {-CUDART_INF_F, 0.f};
      for (uint32_t v = 0; v < R.wholes; v += kStageVecs) {
        uint4 raw[kStageShare];
        take_stage<T>(ring, stage, phase, stages, full, empty, v, R.wholes, waits, ok, raw, KIND == kDistillStep && v >= again);
        uint32_t bits[kStageShare];
        const uint32_t i = R.whole_from + v + tid;
#pragma unroll
        for (int j = 0; j < kStageShare; ++j)  // (behind the row no mark is set, and the room for marks ends with a whole stage)
          bits[j] = listed_of<T>(marks, i + j * kStreamLanes);
        if (__any_sync(kFull, bits[0] | bits[1] | bits[2] | bits[3])) {  // few do: the warp goes around it
#pragma unroll
          for (int j = 0; j < kStageShare; ++j)
            if (bits[j]) drop_elements<T>(raw[j], bits[j]);
        }
        float largest = vec_max<T>(raw[0]);
#pragma unroll
        for (int j = 1; j < kStageShare; ++j) largest = fmaxf(largest, vec_max<T>(raw[j]));
        add_share<T>(raw, largest, c2, acc);
      }
      if (!ok) acc.sum = CUDART_NAN_F;  // a wait has run out: the row is void
      acc = warp_join(acc, c2);
      if (lane == 0) sides[buf].rest[tid >> 5] = acc;
      __syncwarp();
    }
    if (KIND == kDistillLoss) {
      __threadfence_block();
      some_arrive<kStreamLanes + kSideLanes>(kBarDone + buf);
      buf ^= 1;
      continue;
    }
    if (KIND == kDistillStep) {
      some_sync<kStreamLanes>(kBarStream);
      MaxSum rest, all;
      float left;
      w = whole_of(sides[buf], c2, &rest, &all, &left);
    } else {
      w = *reinterpret_cast<const Whole*>(a.stats + row * CVLC_DISTILL_STATS);
    }
    float ca = w.a * (weight / a.temperature);
    unsigned char* const to = reinterpret_cast<unsigned char*>(g) + (int)(R.whole_from * 16) - (int)(R.lead * sizeof(T));  // of the first whole vector
    const bool alike = (reinterpret_cast<uintptr_t>(to) & 15) == 0;
    const uint32_t cuts = (R.wholes + kStageVecs - 1) / kStageVecs, kept = cuts - again / kStageVecs;
    uint32_t held = stage + (stage < kept ? stages : 0) - kept;  // the step: the stage of the first that is held
    for (uint32_t cut = 0; cut < cuts; ++cut) {  // what is held, then the row's beginning
      uint4 raw[kStageShare];
      uint32_t v;
      if (KIND == kDistillStep && cut < kept) {
        v = again + cut * kStageVecs;
        read_stage<T>(ring, held, v, R.wholes, raw);
        release_stage(&empty[held]);
        if (++held == stages) held = 0;
      } else {
        v = (KIND == kDistillStep ? cut - kept : cut) * kStageVecs;
        take_stage<T>(ring, stage, phase, stages, full, empty, v, R.wholes, waits, ok, raw);
      }
      if (!ok) ca = CUDART_NAN_F;
#pragma unroll
      for (int j = 0; j < kStageShare; ++j) {
        float f[E];
        widen<T>(raw[j], f);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 x = __fmul2_rn(__fadd2_rn(make_float2(f[e], f[e + 1]), make_float2(-w.ref, -w.ref)), make_float2(c2, c2));
          const float2 y = __fmul2_rn(make_float2(exp2_fast(x.x), exp2_fast(x.y)), make_float2(ca, ca));
          f[e] = y.x, f[e + 1] = y.y;
        }
        raw[j] = narrow<T>(f);
      }
      const uint32_t i = v + tid;
      if (alike) {
        uint4* const at = reinterpret_cast<uint4*>(to) + i;
        if (v + kStageVecs <= R.wholes) {
#pragma unroll
          for (int j = 0; j < kStageShare; ++j) __stcs(at + j * kStreamLanes, raw[j]);
        } else {
#pragma unroll
          for (int j = 0; j < kStageShare; ++j)
            if (i + j * kStreamLanes < R.wholes) __stcs(at + j * kStreamLanes, raw[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kStageShare; ++j) {
          if (i + j * kStreamLanes >= R.wholes) continue;
          const T* const elements = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
          for (int e = 0; e < E; ++e) reinterpret_cast<T*>(to)[(size_t)(i + j * kStreamLanes) * E + e] = elements[e];
        }
      }
    }
    __threadfence_block();
    some_arrive<kStreamLanes + kSideLanes>(kBarDone + buf);  // the listed words' gradients replace what stands in their places
    buf ^= 1;
  }
}

// how a call's rows are cut: blocks of a cluster for each, threads of a block
struct Cut {
  uint32_t log_blocks, threads, rounds;  // rounds: vectors of a thread at most
  bool few;                              // kFewVecs vectors of a thread hold the block's share
};
constexpr int kFewVecs = 2;  // short shares have more threads instead, each of which is done sooner

// `keep`: most vectors a thread keeps, where the second half works from them (0: it does not).  Blocks of a cluster: as many as keep the row
// (and have room for its marks), and, where rows are few, as many as give every SM two blocks.
Cut cut_rows(const void* logits, uint64_t stride, uint64_t rows, uint32_t vocab, uint32_t size, uint32_t nv, uint32_t keep) {
  const uint32_t per_vec = 16 / size;
  const bool even = (reinterpret_cast<uintptr_t>(logits) & 15) == 0 && stride * size % 16 == 0;  // every row begins with a vector
  const uint32_t vecs = (vocab + per_vec - 1) / per_vec + (even ? 0 : 1), tiles = (vecs + 31) / 32;
  Cut c = {0, 0, 0, false};
  const auto share = [&] { return ((tiles + (1u << c.log_blocks) - 1) >> c.log_blocks) * 32; };
  while (c.log_blocks < 3 && ((keep && share() > keep * kRowThreads) || share() * per_vec > CVLC_MAX_VOCAB / 8)) ++c.log_blocks;
  while (c.log_blocks < 3 && (rows << c.log_blocks) < 2 * kNumSM && (vecs >> c.log_blocks) >= 512) ++c.log_blocks;
  c.few = share() <= kFewVecs * kRowThreads;
  if (c.few) nv = kFewVecs;
  const uint32_t t = ((share() + nv - 1) / nv + 31) & ~31u;
  c.threads = t < 64 ? 64 : (t > kRowThreads ? kRowThreads : t);
  c.rounds = (share() + c.threads - 1) / c.threads;
  return c;
}

// shared memory of a block at most: a bit for every element of an eighth of the longest row, and the most records
constexpr size_t kRowShared = CVLC_MAX_VOCAB / 8 / 8 + 8192 + (size_t)CVLC_MAX_RECORDS * 24;

template <class... Params, class... Args>
cudaError_t launch_rows(int id, void (*kernel)(Params...), uint64_t rows, const Cut& c, bool clusters, size_t smem, cudaStream_t st, Args&&... args) {
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

// Where blocks go from row to row: rows of a few stages each, and so many that a cluster for each of fewer would be slower.  Both sides, us
// (rows of one kernel / of the other): step of 131,072 words bf16, 64 rows 23 / 17, 100 rows 25 / 31, 333 rows 50 / 74; of 32,000 words, 64 rows
// 11 / 9, 100 rows 12 / 15, 1000 rows 43 / 53; of 9000 words, 1000 rows 28 / 22, 4000 rows 98 / 62.
bool streamed(uint64_t rows, uint64_t bytes) { return bytes >= 2 * kStageVecs * 16 && (rows >= kNumSM || (rows >= 80 && bytes >= 3 * kStageVecs * 16)); }
unsigned stream_grid(uint64_t rows) { return (unsigned)(rows < 2 * kNumSM ? rows : 2 * kNumSM); }

template <class T, DistillKind KIND>
cudaError_t distill_typed(const DistillArgs& a, cudaStream_t st) {
  // many long rows: two blocks an SM go from row to row, where two rows' marks and three stages fit
  const uint32_t mark_row = (a.vocab / kPerVec<T> + 2 + kStageVecs) * kPerVec<T> / 128 * 16 + 16;  // the row's, and a stage's behind it
  const size_t beside = 2 * ((size_t)mark_row + records_bytes(a.k));
  if (streamed(a.rows, (uint64_t)a.vocab * sizeof(T)) && beside + 3 * kStageVecs * 16 <= kStreamShared) {
    const uint32_t fit = (uint32_t)((kStreamShared - beside) / (kStageVecs * 16));
    const uint32_t stages = fit < kStagesMost ? fit : kStagesMost;
    const size_t smem = (size_t)stages * kStageVecs * 16 + beside;
    void (*const kernel)(DistillArgs, uint32_t, uint32_t) = k_distill_stream<T, KIND>;
    static OncePerDevice once;
    const cudaError_t e = once_per_device(once, [&] { return allow_shared(kernel, kStreamShared); });
    if (e != cudaSuccess) return e;
    launch_kernel(KIND == kDistillLoss ? kKDistillLoss : KIND == kDistillGrad ? kKDistillGrad : kKDistillStep, kernel,
                  dim3(stream_grid(a.rows)), dim3(kStreamBlock), smem, st, false, a, stages, mark_row);
    return cudaGetLastError();
  }
  constexpr int NV = KIND == kDistillStep ? 8 : 4;
  const Cut c = cut_rows(a.logits, a.row_stride, a.rows, a.vocab, sizeof(T), NV, KIND == kDistillStep ? NV : 0);
  const uint32_t mark_bytes = (c.rounds * c.threads * kPerVec<T> / 8 + 15) & ~15u;  // a bit for every element of a block
  const size_t smem = mark_bytes + records_bytes(a.k);
  void (*const kernel)(DistillArgs, uint32_t, uint32_t) = c.few ? k_distill<T, kFewVecs, KIND> : k_distill<T, NV, KIND>;
  if (smem > 40 * 1024) {  // the most that any call asks for, so that calls of other threads do not matter
    static OncePerDevice once[2];
    const cudaError_t e = smem > kRowShared ? cudaErrorInvalidValue : once_per_device(once[c.few], [&] { return allow_shared(kernel, kRowShared); });
    if (e != cudaSuccess) return e;
  }
  return launch_rows(KIND == kDistillLoss ? kKDistillLoss : KIND == kDistillGrad ? kKDistillGrad : kKDistillStep, kernel, a.rows, c,
                     KIND != kDistillGrad, smem, st, a, c.log_blocks, mark_bytes);
}
// log2(e) / temperature, rounded once
float scale_of(float temperature) { return (float)(1.4426950408889634074 / (double)temperature); }

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
// a thread has loaded, only the largest is looked at first: the k-th largest of the block's thread maxima has at least k elements at or above
// it, and hardly more (a thread rarely holds two).  One block per row goes through it batch by batch, raises that bound as it goes
// (after 1, 2, 4, .. batches and the last) and lists what reaches it: about 3 k elements, of which the last bound leaves little more
// than k.  Those are ranked by (value, word).  Several blocks per row (few rows): the smallest of their bounds for k / blocks each
// serves all of them, and they list from what they have kept.  Rows with more elements at the bound than the lists hold (whole rows
// of equal logits) are selected digit by digit instead.

constexpr uint32_t kTopList = 2048;  // candidates of a row

__device__ __forceinline__ unsigned long long candidate(uint32_t order, uint32_t word) {
  return ((unsigned long long)order << 32) | (uint32_t)~word;
}

constexpr uint32_t kBoundStep = 1u << 15;  // 2^-8 of a value: not worth another round

struct TopPart {
  MaxSum all;
  uint32_t bound;
};

// The largest bound from `lo` on that `want` of the block's threads reach with theirs (`lo` if it is none), to kBoundStep
__device__ __forceinline__ uint32_t raise_bound(uint32_t top, uint32_t want, uint32_t lo, uint32_t* largest) {
  const uint32_t of_warp = __reduce_max_sync(kFull, top);
  if ((threadIdx.x & 31) == 0) atomicMax(largest, of_warp);
  uint32_t n = __syncthreads_count(top >= lo);
  if (n < want) return lo;
  uint32_t hi = *largest;
  __syncthreads();  // all have read it: the next call adds to it
  while (hi > lo && hi - lo > kBoundStep) {
    const uint32_t mid = lo + (hi - lo) / 2;
    n = __syncthreads_count(top >= mid);
    if (n >= want) lo = mid;
    else hi = mid - 1;
    if (n >= want && n <= want + want / 8) break;
  }
  return lo;
}

// element e of a vector, widened
template <class T>
__device__ __forceinline__ float element_of(const uint4& raw, uint32_t e) {
  const uint32_t i = sizeof(T) == 4 ? e : e >> 1;
  const uint32_t w = i & 2 ? (i & 1 ? raw.w : raw.z) : (i & 1 ? raw.y : raw.x);
  if constexpr (sizeof(T) == 4) return __uint_as_float(w);
  const uint16_t h = (uint16_t)(e & 1 ? w >> 16 : w);
  T v;
  memcpy(&v, &h, 2);
  return to_float(v);
}
// bit e: element e of a vector is at least `least`
template <class T>
__device__ __forceinline__ uint32_t reaching(const uint4& raw, float least) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      bits |= __uint_as_float(w[i]) >= least ? 1u << i : 0u;
    } else {  // against the smallest number of the type that is not below `least`
      uint32_t m;
      if constexpr (std::is_same<T, __half>::value) {
        __half2 h;
        memcpy(&h, &w[i], 4);
        m = __hge2_mask(h, __half2half2(__float2half_ru(least)));
      } else {
        __nv_bfloat162 h;
        memcpy(&h, &w[i], 4);
        m = __hge2_mask(h, __bfloat162bfloat162(__float2bfloat16_ru(least)));
      }
      bits |= (m & 0x10001u) << (2 * i);  // the upper one 16 bits above its place
    }
  }
  return sizeof(T) == 4 ? bits : (bits & 0xFFu) | (bits >> 15);
}
// Elements from `least` on (a candidate: value and word) of some vectors, into a list of `room`; word_of(j): the first word of the j-th.
// Few threads have any, and hardly one more than one: they find theirs one by one.
template <class T, class F>
__device__ __forceinline__ void list_vec(const uint4& raw, F&& word_of, unsigned long long least, float floor_value, uint32_t* count,
                                         unsigned long long* to, uint32_t room) {
  for (uint32_t bits = reaching<T>(raw, floor_value); bits; bits &= bits - 1) {
    const uint32_t e = __ffs(bits) - 1;
    const unsigned long long c = candidate(order_of(element_of<T>(raw, e)), (uint32_t)(word_of() + (int)e));
    if (c < least) continue;
    const uint32_t n = atomicAdd(count, 1u);
    if (n < room) to[n] = c;
  }
}
template <class T, int NV, class F>
__device__ __forceinline__ void list_batch(const uint4 (&raw)[NV], F&& word_of, unsigned long long least, uint32_t* count, unsigned long long* to,
                                           uint32_t room) {
  const float floor_value = value_of((uint32_t)(least >> 32));
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (vec_max<T>(raw[j]) >= floor_value) list_vec<T>(raw[j], [&] { return word_of(j); }, least, floor_value, count, to, room);
}

// Digits of the candidates of some vectors that share a prefix, counted; equal ones in a row at once
template <class T>
struct DigitCount {
  uint32_t* hist;
  uint32_t last, run;
  __device__ __forceinline__ void one(float f, uint32_t word, unsigned long long prefix, int shift) {
    if (!(f > -CUDART_INF_F)) return;
    const unsigned long long c = candidate(order_of(f), word);
    if (shift < 56 && (c >> (shift + 8)) != prefix) return;
    const uint32_t digit = (uint32_t)(c >> shift) & 255u;
    if (run && digit != last) {
      atomicAdd(&hist[last], run);
      run = 0;
    }
    last = digit;
    ++run;
  }
  __device__ __forceinline__ void vec(const uint4& raw, int word, unsigned long long prefix, int shift) {
    float f[kPerVec<T>];
    widen<T>(raw, f);
#pragma unroll
    for (int e = 0; e < kPerVec<T>; ++e) one(f[e], (uint32_t)(word + e), prefix, shift);
  }
  __device__ __forceinline__ void done() {
    if (run) atomicAdd(&hist[last], run);
  }
};
// The digit that holds rank `left` from the largest down, and how many lie above it; by a warp, eight digits a lane
template <class F>
__device__ __forceinline__ void pick_digit(F&& count_of, uint32_t left, uint32_t* picked, uint32_t* above) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t n[8], sum = 0;
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    n[d] = count_of(255 - (lane * 8 + d));
    sum += n[d];
  }
  uint32_t before = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(kFull, before, o);
    if (lane >= (uint32_t)o) before += v;
  }
  before -= sum;
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    if (before < left && left <= before + n[d]) *picked = 255 - (lane * 8 + d), *above = before;
    before += n[d];
  }
}

// A row's records from its candidates, whose order is any, by `nt` threads that meet at sync(): `t` is the thread's number.  A record's
// log-probability has two roundings, of the difference and of the result (at a low temperature it is a large number), and is made of halves:
// at a high temperature the difference of two logits may be beyond the type's range and it not.
template <class F>
__device__ __forceinline__ void put_records(const TopArgs& a, uint64_t row, const MaxSum& all, unsigned long long* packed, uint32_t n, uint32_t t,
                                            uint32_t nt, F&& sync) {
  const float ln_sum = logf(all.sum), half_max = 0.5f * all.max;
  auto put = [&](uint32_t at, unsigned long long c) {
    a.ids[row * a.k + at] = (int32_t)~(uint32_t)c;
    const float half = 0.5f * value_of((uint32_t)(c >> 32)) - half_max;
    a.logp[row * a.k + at] = __fmaf_rn(half, a.twice_it, __fmaf_rn(half, a.twice_it_rest, -ln_sum));
  };
  if (n <= 4 * nt) {  // a few for each thread: a candidate's rank is the number of larger ones
    const uint32_t even = (n + 7) & ~7u;
    if (t < even - n) packed[n + t] = 0;
    sync();
    for (uint32_t i = t; i < n; i += nt) {
      const unsigned long long c = packed[i];
      uint32_t larger = 0;
      for (uint32_t o = 0; o < even; o += 8) {
        ulonglong2 p[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = *reinterpret_cast<const ulonglong2*>(packed + o + 2 * q);
#pragma unroll
        for (int q = 0; q < 4; ++q) larger += (p[q].x > c) + (p[q].y > c);
      }
      if (larger < a.k) put(larger, c);
    }
  } else {  // sorted in pairs, the largest first
    uint32_t size = 2;
    while (size < n) size *= 2;
    for (uint32_t i = n + t; i < size; i += nt) packed[i] = 0;
    sync();
    for (uint32_t length = 2; length <= size; length *= 2)
      for (uint32_t apart = length / 2; apart; apart /= 2) {
        for (uint32_t i = t; i < size / 2; i += nt) {
          const uint32_t x = i / apart * 2 * apart + i % apart, y = x + apart;
          const unsigned long long p = packed[x], q = packed[y];
          if ((p < q) == ((x & length) == 0)) packed[x] = q, packed[y] = p;
        }
        sync();
      }
    for (uint32_t i = t; i < a.k && i < n; i += nt) put(i, packed[i]);
  }
  for (uint32_t i = n + t; i < a.k; i += nt) {  // fewer words than records: the others are masked
    a.ids[row * a.k + i] = -1;
    a.logp[row * a.k + i] = -CUDART_INF_F;
  }
}
// ... of a row without a softmax
__device__ __forceinline__ void put_spoiled(const TopArgs& a, uint64_t row, uint32_t t, uint32_t nt) {
  for (uint32_t i = t; i < a.k; i += nt) {
    a.ids[row * a.k + i] = (int32_t)i;
    a.logp[row * a.k + i] = CUDART_NAN_F;
  }
}

template <class T, int NV>
__global__ void __launch_bounds__(kRowThreads, 2) k_top_logits(TopArgs a, uint32_t log_blocks) {
  __shared__ __align__(16) unsigned long long list[kTopList];    // in the first block: a stretch for every block
  __shared__ __align__(16) unsigned long long packed[kTopList];  // the same without gaps
  __shared__ TopPart parts[kMaxClusterBlocks];
  __shared__ MaxSum of_warp[kRowThreads / 32];
  __shared__ uint32_t counts[kMaxClusterBlocks];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t mine, picked, above, largest, kept;
  const uint32_t nt = blockDim.x, tid = threadIdx.x, blocks = 1u << log_blocks, lane = tid & 31, warp_id = tid >> 5;
  const uint32_t rank = blockIdx.x & (blocks - 1);
  const uint64_t row = blockIdx.x >> log_blocks;
  const Row<T> R(a.logits, row, a.row_stride, a.vocab, log_blocks, rank);
  const float c2 = a.c2;
  const uint32_t batches = (R.rounds() + NV - 1) / NV;
  const uint32_t stretch = kTopList >> log_blocks;
  cg::cluster_group cluster = cg::this_cluster();

  uint4 raw[NV];
  load_batch<T, NV>(R, 0, raw);
  if (blocks > 1) cluster_arrive<false>();  // waited for before another block's shared memory is written
  if (tid == 0) mine = largest = kept = 0;
  __syncthreads();

  MaxSum acc = {-CUDART_INF_F, 0.f};
  float low = 0.f;
  uint32_t bound = kOrderNegInf + 1;
  const uint32_t want = (a.k + blocks - 1) >> log_blocks;
  for (uint32_t b = 0;;) {
    uint4 ahead[NV];
    if (b + 1 < batches) load_batch<T, NV>(R, (b + 1) * NV, ahead);
    add_batch<T, NV>(raw, c2, acc, low);
    if (b + 1 == batches || (blocks == 1 && (b & (b + 1)) == 0)) bound = raise_bound(order_of(acc.max), want, bound, &largest);
    if (blocks == 1) list_batch<T, NV>(raw, [&](int j) { return R.word(R.first + (b * NV + j) * R.apart); }, (unsigned long long)bound << 32, &mine, list, stretch);
    if (++b >= batches) break;
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = ahead[j];
  }
  acc.sum += low;
  const MaxSum warp = warp_join(acc, c2);
  if (lane == 0) of_warp[warp_id] = warp;
  __syncthreads();
  MaxSum all = join_warps(of_warp, nt / 32, c2);
  auto relist = [&](unsigned long long least) {  // several blocks, or a second time
    unsigned long long* const to = (blocks > 1 ? cluster.map_shared_rank(list, 0) : list) + rank * stretch;
    for (uint32_t b = 0; b < batches; ++b) {
      if (batches > 1) load_batch<T, NV>(R, b * NV, raw);
      list_batch<T, NV>(raw, [&](int j) { return R.word(R.first + (b * NV + j) * R.apart); }, least, &mine, to, stretch);
    }
    __syncthreads();
    if (tid < blocks) *(blocks > 1 ? cluster.map_shared_rank(&counts[rank], tid) : &counts[rank]) = mine;
    if (blocks > 1) cluster.sync();
    else __syncthreads();
  };
  bool spoiled;  // a NaN or +inf among the logits: there is no softmax
  if (blocks == 1) {
    spoiled = !(all.sum < CUDART_INF_F);
    if (tid == 0) counts[0] = mine;
    __syncthreads();
  } else {
    cluster_wait();
    if (tid < blocks) *cluster.map_shared_rank(&parts[rank], tid) = {all, bound};
    cluster.sync();
    bound = parts[0].bound;
    all = parts[0].all;
    for (uint32_t r = 1; r < blocks; ++r) {
      bound = min(bound, parts[r].bound);
      all = join(all, parts[r].all, c2);
    }
    spoiled = !(all.sum < CUDART_INF_F);
    if (!spoiled) relist((unsigned long long)bound << 32);
  }
  bool overflow = false;
  if (!spoiled)
    for (uint32_t r = 0; r < blocks; ++r) overflow |= counts[r] > stretch;
  if (overflow) {
    // the k-th largest candidate, eight bits at a time
    unsigned long long prefix = 0;
    uint32_t left = a.k;  // rank of the wanted one among those that share the prefix
    for (int shift = 56; shift >= 0; shift -= 8) {
      for (uint32_t i = tid; i < 256; i += nt) hist[i] = 0;
      __syncthreads();
      DigitCount<T> digits = {hist, 0, 0};
      for (uint32_t b = 0; b < batches; ++b) {
        if (batches > 1) load_batch<T, NV>(R, b * NV, raw);
#pragma unroll
        for (int j = 0; j < NV; ++j) digits.vec(raw[j], R.word(R.first + (b * NV + j) * R.apart), prefix, shift);
      }
      digits.done();
      if (blocks > 1) cluster.sync();
      else __syncthreads();
      if (tid < 32)
        pick_digit(
            [&](uint32_t d) {
              uint32_t n = 0;
              for (uint32_t r = 0; r < blocks; ++r) n += (blocks > 1 ? cluster.map_shared_rank(hist, r) : hist)[d];
              return n;
            },
            left, &picked, &above);
      __syncthreads();
      prefix = (prefix << 8) | picked;
      left -= above;
      if (blocks > 1) cluster.sync();  // the counts have been read
      else __syncthreads();
    }
    if (tid == 0) mine = 0;
    __syncthreads();
    relist(prefix);
    bound = (uint32_t)(prefix >> 32);
  }

  if (rank != 0) return;
  if (spoiled) {
    put_spoiled(a, row, tid, nt);
    return;
  }
  // what the last bound leaves, in any order
  for (uint32_t r = 0; r < blocks; ++r) {
    const uint32_t c = counts[r];
    for (uint32_t i = tid; i < c; i += nt) {
      const unsigned long long v = list[r * stretch + i];
      if ((uint32_t)(v >> 32) >= bound) packed[atomicAdd(&kept, 1u)] = v;
    }
  }
  __syncthreads();
  put_records(a, row, all, packed, kept, tid, nt, [] { __syncthreads(); });
}

// Many long rows: as in k_distill_stream, a block goes from row to row, and the side warps rank what the pass over a row has listed while the
// next row is passed over.  (2048 x 131072 bf16, k = 64: a block for every row 200 us, so 139; 82 at the copy bandwidth, 113 without the
// exponentials.)
// What the pass lists is whole vectors, each with its largest element: for a thread of a warp that alone has found one, the elements
// would take many instructions of the whole warp.  The side warps read those again that the last bound leaves.
constexpr uint32_t kSumStages = 32;
constexpr uint32_t kEndWord = 0x80000000u;  // a listed word, not a vector
struct RowTop {
  MaxSum of_warp[kStreamWarps];
  uint32_t count, bound;
};
// LONG: sums of kSumStages stages at a time, since equal terms round the same way (one sum of 1024 stages was off by up to 982 half steps of
// fp32).  Rows of fewer stages do without: 2048 x 131072 bf16 137 us, so 141.
template <class T, bool LONG>
__global__ void __launch_bounds__(kStreamBlock, 2) k_top_stream(TopArgs a, uint32_t stages) {
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ uint64_t full[kStagesMost], empty[kStagesMost];
  __shared__ RowTop tops[2];
  __shared__ uint32_t hist[256];
  static_assert(kStreamLanes == 256, "a bin for each thread");
  __shared__ uint32_t side_hist[256], side_picked, side_above;
  __shared__ uint32_t mine, picked, above, largest, smallest, kept, gone, stopped;
  constexpr int E = kPerVec<T>;
  const uint32_t thread = threadIdx.x, lane = thread & 31;
  const float c2 = a.c2;
  uint4* const ring = reinterpret_cast<uint4*>(dyn);
  unsigned long long* const lists = reinterpret_cast<unsigned long long*>(dyn + (size_t)stages * kStageVecs * 16);  // [2], then the ranking's
  DistillArgs where = {};
  where.logits = a.logits, where.row_stride = a.row_stride, where.vocab = a.vocab;
  const Waits waits = {&gone, &stopped, nullptr, kWaitMost};

  if (thread == 0) {
    for (uint32_t i = 0; i < stages; ++i) bar_init(&full[i], 1), bar_init(&empty[i], kStreamWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    mine = kept = gone = stopped = 0;
  }
  __syncthreads();
  bool ok = true;
  if (thread >= kSideLanes && thread < kStreamFirst) {
    if (lane == 0) copy_rows<T, 1>(where, a.rows, ring, stages, full, empty, waits, [](uint64_t) { return false; });
    return;
  }
  if (thread < kSideLanes) {
    const uint32_t t = thread;
    unsigned long long* const packed = lists + 2 * kTopList;
    uint32_t buf = 0;
    some_arrive<kStreamLanes + kSideLanes>(kBarReady);
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, buf ^= 1) {
      if (row + gridDim.x < a.rows) some_arrive<kStreamLanes + kSideLanes>(kBarReady + (buf ^ 1));  // the next row's list is free
      some_sync<kStreamLanes + kSideLanes>(kBarDone + buf);
      const RowTop& s = tops[buf];
      const MaxSum all = join_warps(s.of_warp, kStreamWarps, c2);
      if (!(all.sum < CUDART_INF_F)) {
        put_spoiled(a, row, t, kSideLanes);
      } else {
        const unsigned long long* const list = lists + buf * kTopList;
        const uint32_t c = s.count;
        uint32_t bound = s.bound;
        if (c > a.k) {  // the k-th largest of what is listed, to a bin, is the last bound
          for (uint32_t i = t; i < 256; i += kSideLanes) side_hist[i] = 0;
          some_sync<kSideLanes>(kBarSide);
          const uint32_t hi = max(order_of(all.max), bound), shift = hi > bound ? max(24 - __clz(hi - bound), 0) : 0;
          for (uint32_t i = t; i < c; i += kSideLanes) {
            const uint32_t order = (uint32_t)(list[i] >> 32);
            if (order >= bound) atomicAdd(&side_hist[min((order - bound) >> shift, 255u)], 1u);
          }
          some_sync<kSideLanes>(kBarSide);
          if (t < 32) {
            if (t == 0) side_picked = 0;
            __syncwarp();
            pick_digit([&](uint32_t d) { return side_hist[d]; }, a.k, &side_picked, &side_above);
          }
          some_sync<kSideLanes>(kBarSide);
          bound += side_picked << shift;
        }
        const RowAt R = row_at<T>(where, row);
        const uint4* const from = reinterpret_cast<const uint4*>(R.from) + R.whole_from;
        // f(value, word) of every listed element
        const auto each = [&](auto&& f) {
          for (uint32_t i = t; i < c; i += kSideLanes) {
            const uint32_t order = (uint32_t)(list[i] >> 32), id = (uint32_t)list[i];
            if (order < bound) continue;
            if (id & kEndWord) {
              f(value_of(order), id & ~kEndWord);
            } else {
              float v[E];
              widen<T>(__ldg(from + id), v);
              const int word = (int)((R.whole_from + id) * E) - (int)R.lead;
#pragma unroll
              for (int e = 0; e < E; ++e) f(v[e], (uint32_t)(word + e));
            }
          }
        };
        const auto keep = [&](unsigned long long least) {
          each([&](float v, uint32_t word) {
            if (!(v >= value_of((uint32_t)(least >> 32)))) return;
            const unsigned long long x = candidate(order_of(v), word);
            if (x < least) return;
            const uint32_t n = atomicAdd(&kept, 1u);
            if (n < kTopList) packed[n] = x;
          });
          some_sync<kSideLanes>(kBarSide);
        };
        keep((unsigned long long)bound << 32);
        if (kept > kTopList) {  // equal elements in many of the vectors: the k-th largest among them, eight bits at a time
          unsigned long long prefix = 0;
          uint32_t left = a.k;
          for (int shift = 56; shift >= 0; shift -= 8) {
            for (uint32_t i = t; i < 256; i += kSideLanes) side_hist[i] = 0;
            some_sync<kSideLanes>(kBarSide);
            DigitCount<T> digits = {side_hist, 0, 0};
            each([&](float v, uint32_t word) { digits.one(v, word, prefix, shift); });
            digits.done();
            some_sync<kSideLanes>(kBarSide);
            if (t < 32) pick_digit([&](uint32_t d) { return side_hist[d]; }, left, &side_picked, &side_above);
            some_sync<kSideLanes>(kBarSide);
            prefix = (prefix << 8) | side_picked;
            left -= side_above;
          }
          some_sync<kSideLanes>(kBarSide);
          if (t == 0) kept = 0;
          some_sync<kSideLanes>(kBarSide);
          keep(prefix);
        }
        put_records(a, row, all, packed, kept, t, kSideLanes, [] { some_sync<kSideLanes>(kBarSide); });
        some_sync<kSideLanes>(kBarSide);
        if (t == 0) kept = 0;
      }
      some_sync<kSideLanes>(kBarSide);
    }
    return;
  }

  const uint32_t tid = thread - kStreamFirst;
  uint32_t stage = 0, phase = 0, buf = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, buf ^= 1) {
    const RowAt R = row_at<T>(where, row);
    const T* const z = reinterpret_cast<const T*>(R.from) + R.lead;
    const int end = end_word<E>(R, a.vocab, tid);  // ends of the row beside its whole vectors: one for a thread
    const float end_z = end >= 0 ? to_float(z[end]) : -CUDART_INF_F;
    some_sync<kStreamLanes + kSideLanes>(kBarReady + buf);
    if (tid == 0) mine = 0, largest = 0, smallest = 0xFFFFFFFFu;
    hist[tid] = 0;
    some_sync<kStreamLanes>(kBarStream);
    unsigned long long* const list = lists + buf * kTopList;
    MaxSum acc = {end_z, end_z == -CUDART_INF_F ? 0.f : end_z < CUDART_INF_F ? 1.f : CUDART_NAN_F};
    if (end_z != end_z) acc.max = -CUDART_INF_F;
    // after 1, 4, 16, .. stages, which lists about 7 k vectors; after 1, 2, 4, .. where that could be too many
    const uint32_t often = a.k <= 96 ? 4 : 2;
    float top[2] = {-CUDART_INF_F, -CUDART_INF_F};  // the thread's largest, of every other vector
    uint32_t bound = kOrderNegInf + 1, next_raise = 0;
    const uint32_t cuts = (R.wholes + kStageVecs - 1) / kStageVecs;
    MaxSum earlier = {-CUDART_INF_F, 0.f};
    const auto note = [&](uint32_t order, uint32_t id) {
      const uint32_t n = atomicAdd(&mine, 1u);
      if (n < kTopList) list[n] = (unsigned long long)order << 32 | id;
    };
    for (uint32_t b = 0; b < cuts; ++b) {
      uint4 raw[kStageShare];
      take_stage<T>(ring, stage, phase, stages, full, empty, b * kStageVecs, R.wholes, waits, ok, raw);
      float largest_of[kStageShare];
#pragma unroll
      for (int j = 0; j < kStageShare; ++j) largest_of[j] = vec_max<T>(raw[j]), top[j & 1] = fmaxf(top[j & 1], largest_of[j]);
      const float top_of = fmaxf(fmaxf(largest_of[0], largest_of[1]), fmaxf(largest_of[2], largest_of[3]));
      add_share<T>(raw, top_of, c2, acc);
      if (LONG && (b + 1) % kSumStages == 0) {
        earlier = join(earlier, acc, c2);
        acc.sum = 0.f;
      }
      if (b == next_raise && b + 1 < cuts) {
        // The bound is raised by a histogram of the threads' maxima (two of a thread) between the last bound (at first: the smallest of
        // them) and the largest
        next_raise = next_raise * often + often - 1;
        const uint32_t mine_of[2] = {order_of(top[0]), order_of(top[1])};
        const uint32_t most = __reduce_max_sync(kFull, max(mine_of[0], mine_of[1])), least = __reduce_min_sync(kFull, min(mine_of[0], mine_of[1]));
        if (lane == 0) atomicMax(&largest, most), atomicMin(&smallest, least);
        some_sync<kStreamLanes>(kBarStream);
        uint32_t lo = b ? bound : max(smallest, kOrderNegInf + 1), hi = largest, left = a.k;
        while (true) {
          const uint32_t shift = hi > lo ? max(24 - __clz(hi - lo), 0) : 0;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (mine_of[h] >= lo && mine_of[h] <= hi) atomicAdd(&hist[(mine_of[h] - lo) >> shift], 1u);
          some_sync<kStreamLanes>(kBarStream);
          if (tid < 32) {
            if (tid == 0) picked = 0, above = 0;  // fewer than k: the lowest bin
            __syncwarp();
            pick_digit([&](uint32_t d) { const uint32_t n = hist[d]; hist[d] = 0; return n; }, left, &picked, &above);
          }
          some_sync<kStreamLanes>(kBarStream);
          lo += picked << shift;
          if (shift <= 18) break;
          hi = lo + ((1u << shift) - 1), left -= above;  // a bin of more than 1 / 32 of an octave: its own histogram
        }
        bound = lo;
      }
      const float floor_value = value_of(bound);
      if (__any_sync(kFull, top_of >= floor_value)) {  // the warp goes around what none of its threads has
#pragma unroll
        for (int j = 0; j < kStageShare; ++j)
          if (largest_of[j] >= floor_value) note(order_of(largest_of[j]), b * kStageVecs + tid + j * kStreamLanes);
      }
    }
    if (end_z >= value_of(bound)) note(order_of(end_z), kEndWord | (uint32_t)end);
    if (!ok) acc.sum = CUDART_NAN_F;  // a wait has run out: the row is void
    if (LONG) acc = join(earlier, acc, c2);
    const MaxSum warp = warp_join(acc, c2);
    if (lane == 0) tops[buf].of_warp[tid >> 5] = warp;
    some_sync<kStreamLanes>(kBarStream);
    if (mine > kTopList) {
      // the k-th largest candidate, eight bits at a time, read again from global memory
      unsigned long long prefix = 0;
      uint32_t left = a.k;
      const uint4* const from = reinterpret_cast<const uint4*>(R.from) + R.whole_from;
      for (int shift = 56; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        some_sync<kStreamLanes>(kBarStream);
        DigitCount<T> digits = {hist, 0, 0};
        for (uint32_t i = tid; i < R.wholes; i += kStreamLanes)
          digits.vec(__ldg(from + i), (int)((R.whole_from + i) * E) - (int)R.lead, prefix, shift);
        digits.one(end_z, (uint32_t)end, prefix, shift);
        digits.done();
        some_sync<kStreamLanes>(kBarStream);
        if (tid < 32) pick_digit([&](uint32_t d) { return hist[d]; }, left, &picked, &above);
        some_sync<kStreamLanes>(kBarStream);
        prefix = (prefix << 8) | picked;
        left -= above;
      }
      some_sync<kStreamLanes>(kBarStream);
      if (tid == 0) mine = 0;
      some_sync<kStreamLanes>(kBarStream);
      // its k candidates stand in the list as words
      const float floor_value = value_of((uint32_t)(prefix >> 32));
      for (uint32_t i = tid; i < R.wholes; i += kStreamLanes) {
        const uint4 raw = __ldg(from + i);
        const int word = (int)((R.whole_from + i) * E) - (int)R.lead;
        for (uint32_t bits = reaching<T>(raw, floor_value); bits; bits &= bits - 1) {
          const uint32_t e = __ffs(bits) - 1, order = order_of(element_of<T>(raw, e));
          if (candidate(order, (uint32_t)(word + (int)e)) >= prefix) note(order, kEndWord | (uint32_t)(word + (int)e));
        }
      }
      if (end_z > -CUDART_INF_F && candidate(order_of(end_z), (uint32_t)end) >= prefix) note(order_of(end_z), kEndWord | (uint32_t)end);
      bound = (uint32_t)(prefix >> 32);
      some_sync<kStreamLanes>(kBarStream);
    }
    if (tid == 0) tops[buf].count = min(mine, kTopList), tops[buf].bound = bound;
    __threadfence_block();
    some_arrive<kStreamLanes + kSideLanes>(kBarDone + buf);
  }
}

// The ring alone, one block: `give_back`: a thread takes the row's stages and gives them back; else none is given back, and the copies stop
// when the wait for one has run out.  seen: what the stages hold then.
constexpr uint32_t kSelftestStages = 2;
__global__ void k_selftest_ring(DistillArgs a, int32_t* status, uint64_t most, int give_back, uint4* seen) {
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ uint64_t full[kSelftestStages], empty[kSelftestStages];
  __shared__ uint32_t gone, stopped;
  uint4* const ring = reinterpret_cast<uint4*>(dyn);
  const Waits waits = {&gone, &stopped, status, most};
  if (threadIdx.x == 0) {
    gone = stopped = 0;
    for (uint32_t i = 0; i < kSelftestStages; ++i) bar_init(&full[i], 1), bar_init(&empty[i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (threadIdx.x == 0) copy_rows<float, 1>(a, 1, ring, kSelftestStages, full, empty, waits, [](uint64_t) { return false; });
  if (threadIdx.x >= 32 && threadIdx.x < 64) {
    const uint32_t cuts = a.vocab / (kStageVecs * kPerVec<float>);
    bool ok = true;
    for (uint32_t c = 0; c < cuts; ++c) {
      bar_wait(&full[c % kSelftestStages], c / kSelftestStages & 1, waits, ok);
      if (give_back) release_stage(&empty[c % kSelftestStages]);
    }
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < kSelftestStages * kStageVecs; i += blockDim.x) seen[i] = ring[i];
}

template <class T>
cudaError_t top_typed(const TopArgs& a, cudaStream_t st) {
  if (streamed(a.rows, (uint64_t)a.vocab * sizeof(T))) {
    const size_t beside = 3 * kTopList * 8;
    const uint32_t stages = (uint32_t)((kStreamShared - beside) / (kStageVecs * 16));
    const size_t smem = (size_t)stages * kStageVecs * 16 + beside;
    const bool more = (uint64_t)a.vocab * sizeof(T) > (uint64_t)kSumStages * kStageVecs * 16;
    void (*const kernel)(TopArgs, uint32_t) = more ? k_top_stream<T, true> : k_top_stream<T, false>;
    static OncePerDevice once[2];
    const cudaError_t e = once_per_device(once[more], [&] { return allow_shared(kernel, kStreamShared); });
    if (e != cudaSuccess) return e;
    launch_kernel(kKTopLogits, kernel, dim3(stream_grid(a.rows)), dim3(kStreamBlock), smem, st, false, a, stages);
    return cudaGetLastError();
  }
  constexpr int NV = 4;
  Cut c = cut_rows(a.logits, a.row_stride, a.rows, a.vocab, sizeof(T), NV, 0);
  // the bound is the better the more threads the row's elements are spread over
  while (c.threads < kRowThreads && c.threads < 2 * (a.k >> c.log_blocks) && c.rounds > 1) {
    const uint32_t held = c.rounds * c.threads;
    c.threads += 32;
    c.rounds = (held + c.threads - 1) / c.threads;
  }
  void (*const kernel)(TopArgs, uint32_t) = c.few ? k_top_logits<T, kFewVecs> : k_top_logits<T, NV>;
  return launch_rows(kKTopLogits, kernel, a.rows, c, true, 0, st, a, c.log_blocks);
}

}  // namespace

cudaError_t launch_selftest_ring(const float* row, uint32_t cuts, int give_back, uint64_t most, int32_t* status, float* seen, cudaStream_t st) {
  DistillArgs a = {};
  a.logits = row, a.rows = 1, a.vocab = cuts * kStageVecs * kPerVec<float>, a.row_stride = a.vocab;
  LaunchScope ls(kKSelftest, st);
  k_selftest_ring<<<1, 64, kSelftestStages * kStageVecs * 16, st>>>(a, status, most, give_back, reinterpret_cast<uint4*>(seen));
  return cudaGetLastError();
}

cudaError_t launch_top_logits(const TopArgs& args, uint32_t dtype, cudaStream_t st) {
  TopArgs a = args;
  a.c2 = scale_of(a.temperature);
  const double twice_it = 2.0 / (double)a.temperature;
  a.twice_it = (float)twice_it;
  a.twice_it_rest = (float)(twice_it - (double)a.twice_it);
  if (dtype == CVLC_F32) return top_typed<float>(a, st);
  if (dtype == CVLC_F16) return top_typed<__half>(a, st);
  return top_typed<__nv_bfloat16>(a, st);
}

cudaError_t launch_distill(const DistillArgs& args, uint32_t dtype, DistillKind kind, cudaStream_t st) {
  DistillArgs a = args;
  a.c2 = scale_of(a.temperature);
  if (dtype == CVLC_F32) return distill_kind<float>(a, kind, st);
  if (dtype == CVLC_F16) return distill_kind<__half>(a, kind, st);
  return distill_kind<__nv_bfloat16>(a, kind, st);
}

}  // namespace cvlc
