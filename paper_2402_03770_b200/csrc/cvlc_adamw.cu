// AdamW over many tensors at once, with states in fp32 or in 8 bits, and the norm of their gradients.
//
// m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p -= lr (wd p + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
//
// Nothing is used twice, so the step is bounded by what it moves: 30 bytes a value with fp32 weights and states, bf16 gradients and a bf16
// copy, 16 with states of 8 bits.  All tensors go in one launch: their descriptors are a parameter of the kernel, a block finds its tensor by
// the number of its first chunk.  A warp has 256 values at a time, 8 consecutive ones a lane: the values that share a scale, so that their
// largest is found by one reduction of a warp and the states are read and written once.
#include "cvlc_common.cuh"
#include "cvlc_vocab.cuh"

namespace cvlc {
namespace {

constexpr int kBlock = CVLC_STATE_BLOCK;  // values of a warp at a time, and of a scale
constexpr int kPer = kBlock / 32;         // consecutive ones of a lane
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kNormChunks = 24 * kNumSM;  // of the norm, at most, and one more for every tensor

// Which of a tensor's arrays can be read and written by vectors.  fp32 states have no blocks of their own, so that their tensors are cut where the
// weights' addresses are multiples of 32 bytes: `lead` values before the first are not there.
enum : uint32_t { kVecParam = 1, kVecGrad = 2, kVecM = 4, kVecV = 8, kVecCopy = 16 };
struct TensorDesc {
  uint64_t n;
  const void* grad;
  void *param, *m, *v, *copy;
  float2* scale;
  float lr, decay;
  uint32_t first;  // its first chunk
  uint16_t vec, lead;
};
struct StepScalars {
  float lr, b1, b1r, b2, b2r, eps, ic1, ic2, grad_scale, max_norm;  // ic: 1 / (1 - beta^t), the second 2^24 times that
  double beta1, beta2;
  const float *norm, *lr_dev;
  const uint32_t* step_dev;
  uint64_t seed;
  uint32_t step, chunk;  // blocks of values in a chunk
  uint32_t param_dtype, grad_dtype, copy_dtype;
  uint32_t tensor0;  // number of the first tensor of this launch
  int32_t* status;
};
// Launch parameters cost the host what they hold (24 KB about 3 us), so there are three capacities.
constexpr uint32_t kFew = 8, kSome = 64, kMany = 440;
template <uint32_t CAP>
struct TensorList {
  uint32_t n, chunks;
  StepScalars s;
  TensorDesc t[CAP];
};
static_assert(sizeof(TensorList<kMany>) <= 32764, "launch parameters");

template <uint32_t CAP>
__device__ __forceinline__ uint32_t tensor_of(const TensorList<CAP>& L, uint32_t chunk) {
  uint32_t lo = 0, hi = L.n;  // the last one whose first chunk is not behind it
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (L.t[mid].first <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

// Eight values from `at` on, in two steps, so that the loads of all arrays are on their way before the first value is used.  Those outside of [0, n) are 0
// and are not touched.
struct Raw {
  uint4 a, b;  // b: of fp32 only
};
__device__ __forceinline__ uint4 scalars16(const uint16_t* p, int64_t at, uint64_t n) {
  uint32_t x[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = (uint64_t)(at + i) < n ? p[i] : 0u;
  return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
}
__device__ __forceinline__ Raw fetch8(bool f32, const void* base, int64_t at, uint64_t n, bool vec) {
  Raw r;
  if (f32) {
    const uint32_t* const p = static_cast<const uint32_t*>(base) + at;
    if (vec) {
      r.a = __ldcs(reinterpret_cast<const uint4*>(p)), r.b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
    } else {
      uint32_t x[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = (uint64_t)(at + i) < n ? p[i] : 0u;
      r.a = make_uint4(x[0], x[1], x[2], x[3]), r.b = make_uint4(x[4], x[5], x[6], x[7]);
    }
  } else {
    const uint16_t* const p = static_cast<const uint16_t*>(base) + at;
    r.a = vec ? __ldcs(reinterpret_cast<const uint4*>(p)) : scalars16(p, at, n);
    r.b = make_uint4(0, 0, 0, 0);
  }
  return r;
}
__device__ __forceinline__ void widen8(uint32_t dtype, const Raw& r, float (&x)[kPer]) {
  if (dtype == CVLC_F32) {
    float y[4], z[4];
    widen<float>(r.a, y), widen<float>(r.b, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i], x[4 + i] = z[i];
  } else if (dtype == CVLC_F16) {
    widen<__half>(r.a, x);
  } else {
    widen<__nv_bfloat16>(r.a, x);
  }
}
template <class T>
__device__ __forceinline__ void store8(void* base, int64_t at, uint64_t n, bool vec, const float (&x)[kPer]) {
  T* p = static_cast<T*>(base) + at;
  if (vec) {
    constexpr int per = kPerVec<T>;
#pragma unroll
    for (int i = 0; i < kPer / per; ++i) {
      float y[per];
#pragma unroll
      for (int k = 0; k < per; ++k) y[k] = x[i * per + k];
      __stcs(reinterpret_cast<uint4*>(p) + i, narrow<T>(y));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if ((uint64_t)(at + i) < n) p[i] = from_float<T>(x[i]);
  }
}
__device__ __forceinline__ void store8(uint32_t dtype, void* base, int64_t at, uint64_t n, bool vec, const float (&x)[kPer]) {
  if (dtype == CVLC_F32) store8<float>(base, at, n, vec, x);
  else if (dtype == CVLC_F16) store8<__half>(base, at, n, vec, x);
  else store8<__nv_bfloat16>(base, at, n, vec, x);
}
__device__ __forceinline__ uint2 fetch_bytes(const void* base, int64_t at, uint64_t n, bool vec) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + at;
  if (vec) return __ldcs(reinterpret_cast<const uint2*>(p));
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if ((uint64_t)(at + i) < n) w[i / 4] |= (uint32_t)p[i] << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_bytes(void* base, int64_t at, uint64_t n, bool vec, const uint32_t (&w)[2]) {
  uint8_t* p = static_cast<uint8_t*>(base) + at;
  if (vec) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
    return;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if ((uint64_t)(at + i) < n) p[i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
}

// ---- 8-bit states --------------------------------------------------------------------------
// m is held in e4m3 (largest value 448), v in e5m2 (57344), relative to the largest value of the block of 256.  A float's bits are linear
// between two neighbouring values of the short type, so rounding up with the probability of what is cut off is adding random bits below the cut.
// Rounding to nearest would not do: an average that moves by a thousandth a step never leaves a value whose neighbours are an eighth away.
// Times a power of two that brings the type's smallest normal value to fp32's, the code is the float's upper bits, subnormal values included
// (their product is rounded at 2^-29 of the type's 1).  y, from 0 up, becomes its code in the upper byte of a word, moved there with the addition;
// `random`: 16 random bits above half of what they tell apart.
template <int MANTISSA>
__device__ __forceinline__ uint32_t to_float8(float y, uint32_t random) {
  constexpr float most = MANTISSA == 3 ? 448.0f : 57344.0f, bias = MANTISSA == 3 ? 0x1p-120f : 0x1p-112f;
  return __float_as_uint(fminf(y, most) * bias) * (MANTISSA == 3 ? 16u : 8u) + random;
}
__device__ __forceinline__ uint32_t upper_bytes(const uint32_t (&x)[4]) {
  return __byte_perm(__byte_perm(x[0], x[1], 0x0073), __byte_perm(x[2], x[3], 0x0073), 0x5410);
}
// bit 7 of every byte whose lower seven bits are not all 0
__device__ __forceinline__ uint32_t some_bits(uint32_t w) { return (w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu; }
// the largest of three sizes; what is not a number stays that
__device__ __forceinline__ float largest(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
  return r;
}
// Four codes as floats: e4m3 by way of fp16, which holds all its values; e5m2 is the upper half of an fp16
__device__ __forceinline__ void from_e4m3(uint32_t w, float (&x)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t y;
    asm("{.reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.rn.f16x2.e4m3x2 %0, a;}" : "=r"(y) : "r"(w >> (16 * h)));
    __half2 z;
    memcpy(&z, &y, 4);
    const float2 f = __half22float2(z);
    x[2 * h] = f.x, x[2 * h + 1] = f.y;
  }
}
__device__ __forceinline__ void from_e5m2(uint32_t w, float (&x)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t y = __byte_perm(w, 0, h ? 0x3424 : 0x1404);
    __half2 z;
    memcpy(&z, &y, 4);
    const float2 f = __half22float2(z);
    x[2 * h] = f.x, x[2 * h + 1] = f.y;
  }
}
// all four words of a counter, the round keys worked out once
__device__ __forceinline__ uint4 philox4x32_10(uint4 c, const PhiloxRoundKeys& rk) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const unsigned long long p0 = (unsigned long long)0xD2511F53u * c.x, p1 = (unsigned long long)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(p1 >> 32) ^ c.y ^ rk.x[i], (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c.w ^ rk.y[i], (uint32_t)p0);
  }
  return c;
}
constexpr float kLeast = 0x1p-100f;  // a block whose largest value is below this is held as zeros

// Threads of a block: with 8-bit states a block of 128 needs fewer registers a thread (48, 61 of 256), and 40 warps share an SM (100 M values: 324 -> 299 us);
// with 32 bits the loads alone fill it (11 M values in one vector 73 and 78).
template <bool EIGHT>
constexpr int kStepThreads = EIGHT ? 128 : 256;
template <bool EIGHT, uint32_t CAP>
__global__ void __launch_bounds__(kStepThreads<EIGHT>) k_adamw(const __grid_constant__ TensorList<CAP> L) {
  const StepScalars& s = L.s;
  __shared__ float corrections[2];
  float ic1 = s.ic1, ic2 = s.ic2;
  uint32_t step = s.step;
  if (s.step_dev) {
    step = *s.step_dev;
    if (step == 0) {  // the averages have nothing to be divided by
      if (s.status && blockIdx.x == 0 && threadIdx.x == 0) set_status(s.status, CVLC_ERR_INVALID_ARG);
      return;
    }
    if (threadIdx.x == 0) {
      double p1 = 1.0, p2 = 1.0, q1 = s.beta1, q2 = s.beta2;
      for (uint32_t k = step; k; k >>= 1) {
        if (k & 1) p1 *= q1, p2 *= q2;
        q1 *= q1, q2 *= q2;
      }
      corrections[0] = (float)(1.0 / (1.0 - p1)), corrections[1] = (float)(0x1p24 / (1.0 - p2));
    }
    __syncthreads();
    ic1 = corrections[0], ic2 = corrections[1];
  }
  float scale = s.grad_scale;
  if (s.norm) {
    const float norm = *s.norm;
    if (!(norm < CUDART_INF_F)) {  // nothing is to be learnt from such gradients
      if (s.status && blockIdx.x == 0 && threadIdx.x == 0) set_status(s.status, CVLC_ERR_NONFINITE_INPUT);
      return;
    }
    scale *= norm > s.max_norm ? s.max_norm / norm : 1.0f;
  }
  const uint32_t index = tensor_of(L, blockIdx.x);
  const TensorDesc& t = L.t[index];
  const PhiloxRoundKeys keys = philox_round_keys(s.seed);
  const float lr = (s.lr_dev ? s.lr * *s.lr_dev : s.lr) * t.lr;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const uint64_t blocks = (t.n + t.lead + kBlock - 1) / kBlock;
  uint64_t block = (uint64_t)(blockIdx.x - t.first) * s.chunk + warp;
  const uint64_t end = min(blocks, (uint64_t)(blockIdx.x - t.first + 1) * s.chunk);
  for (; block < end; block += kStepThreads<EIGHT> / 32) {
    const int64_t at = (int64_t)(block * kBlock + lane * kPer) - t.lead;
    const uint32_t vec = at >= 0 && (uint64_t)at + kPer <= t.n ? t.vec : 0;
    float p[kPer], g[kPer], m[kPer], v[kPer];
    const Raw rp = fetch8(s.param_dtype == CVLC_F32, t.param, at, t.n, vec & kVecParam), rg = fetch8(s.grad_dtype == CVLC_F32, t.grad, at, t.n, vec & kVecGrad);
    if (EIGHT) {
      const uint2 cm = fetch_bytes(t.m, at, t.n, vec & kVecM), cv = fetch_bytes(t.v, at, t.n, vec & kVecV);
      const float2 sc = __ldcs(t.scale + block);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[4], y[4];
        from_e4m3(h ? cm.y : cm.x, x);
        from_e5m2(h ? cv.y : cv.x, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[4 * h + i] = x[i] * sc.x, v[4 * h + i] = y[i] * sc.y;
      }
    } else {
      const Raw rm = fetch8(true, t.m, at, t.n, vec & kVecM), rv = fetch8(true, t.v, at, t.n, vec & kVecV);
      widen8(CVLC_F32, rm, m), widen8(CVLC_F32, rv, v);
    }
    widen8(s.param_dtype, rp, p), widen8(s.grad_dtype, rg, g);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      // every product and sum is rounded by itself, in this order: what an 8-bit state becomes is then a function of its inputs' bits
      const float x = g[i] * scale;
      m[i] = s.b1 * m[i] + s.b1r * x;
      v[i] = s.b2 * v[i] + s.b2r * (x * x);
      // the root's argument is raised by 2^24, so that no v is flushed to 0 (above 2^104 it becomes infinite, and the step 0)
      float root, inverse;
      asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(v[i] * ic2));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(fmaf(root, 0x1p-12f, s.eps)));  // of 1e-30 or more
      p[i] = fmaf(-lr, fmaf(t.decay, p[i], m[i] * ic1 * inverse), p[i]);
    }
    store8(s.param_dtype, t.param, at, t.n, vec & kVecParam, p);
    if (t.copy) {  // of the weights as they are held
      if (s.param_dtype != CVLC_F32)
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = s.param_dtype == CVLC_F16 ? to_float(from_float<__half>(p[i])) : to_float(from_float<__nv_bfloat16>(p[i]));
      if (s.copy_dtype == CVLC_F16) store8<__half>(t.copy, at, t.n, vec & kVecCopy, p);
      else store8<__nv_bfloat16>(t.copy, at, t.n, vec & kVecCopy, p);
    }
    if (EIGHT) {
      float am = 0.0f, av = 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; i += 2) am = largest(am, m[i], m[i + 1]), av = largest(av, v[i], v[i + 1]);
      const float a = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(am))), b = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(av)));
      const float inverse = 1.0f / (lane & 16 ? b : a), of_a = __shfl_sync(kFull, inverse, 0), of_b = __shfl_sync(kFull, inverse, 16);  // one division for both
      const float ia = a >= kLeast ? 448.0f * of_a : 0.0f, ib = b >= kLeast ? 57344.0f * of_b : 0.0f;
      const uint64_t quad = (uint64_t)at / 4;
      uint32_t wm[2], wv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 r = philox4x32_10(make_uint4((uint32_t)(quad + h), (uint32_t)((quad + h) >> 32), s.tensor0 + index, step), keys);
        const uint32_t word[4] = {r.x, r.y, r.z, r.w};
        uint32_t c[4], d[4];
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = m[4 * h + i];
          y[i] = v[4 * h + i] * ib;
          c[i] = (to_float8<3>(fabsf(x) * ia, __byte_perm(word[i], 0x80, 0x5104)) & 0x7FFFFFFFu) | (__float_as_uint(x) & 0x80000000u);
          d[i] = to_float8<2>(y[i], __byte_perm(word[i], 0x80, 0x5324));
        }
        wm[h] = upper_bytes(c);
        wm[h] &= some_bits(wm[h]) | 0x7F7F7F7Fu;  // 0 has no sign
        // a second moment that is there never becomes 0: the step would divide by eps alone (asked of v itself: next to one 2^166 times as large y is 0)
        if ((some_bits(upper_bytes(d)) & 0x80808080u) != 0x80808080u) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (d[i] < 1u << 24) d[i] = v[4 * h + i] > 0.0f && ib > 0.0f ? 1u << 24 : 0u;
        }
        wv[h] = upper_bytes(d);
      }
      store_bytes(t.m, at, t.n, vec & kVecM, wm);
      store_bytes(t.v, at, t.n, vec & kVecV, wv);
      // 0 for a block of zeros; what is not a number stays that
      if (lane == 0) __stcs(t.scale + block, make_float2(a < kLeast ? 0.0f : a * (1.0f / 448.0f), b < kLeast ? 0.0f : b * (1.0f / 57344.0f)));
    } else {
      store8<float>(t.m, at, t.n, vec & kVecM, m);
      store8<float>(t.v, at, t.n, vec & kVecV, v);
    }
  }
}

// ---- norm ----------------------------------------------------------------------------------
// Squares of a lane's 8 values in 32 bits, their sums in 64: the result is right to a rounding and does not depend on the order of blocks.
__device__ __forceinline__ double sum_of_block(double x, double* shared) {
#pragma unroll
  for (int d = 16; d; d /= 2) x += __shfl_xor_sync(kFull, x, d);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
  __syncthreads();
  x = 0.0;
  for (int i = 0; i < (int)blockDim.x / 32; ++i) x += shared[i];
  return x;
}
template <uint32_t CAP>
__global__ void __launch_bounds__(kThreads) k_norm_parts(const __grid_constant__ TensorList<CAP> L, double* parts) {
  __shared__ double shared[kWarps];
  const StepScalars& s = L.s;
  const TensorDesc& t = L.t[tensor_of(L, blockIdx.x)];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31, chunk = blockIdx.x - t.first;
  const uint64_t blocks = (t.n + t.lead + kBlock - 1) / kBlock, begin = (uint64_t)chunk * s.chunk;
  const uint32_t mine = (uint32_t)min((uint64_t)s.chunk, blocks - begin);  // blocks of values of this block of threads
  const int64_t from = (int64_t)(begin * kBlock + lane * kPer) - t.lead;
  constexpr int kAhead = 4;  // loads of a thread that are on their way together
  double sum = 0.0;
  for (uint32_t b = warp; b < mine; b += kAhead * kWarps) {
    Raw r[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t at = from + (int64_t)(b + k * kWarps) * kBlock;
      const uint64_t n = b + k * kWarps < mine ? t.n : 0;
      r[k] = fetch8(s.grad_dtype == CVLC_F32, t.grad, at, n, (t.vec & kVecGrad) && at >= 0 && (uint64_t)at + kPer <= n);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float g[kPer], q = 0.0f;
      widen8(s.grad_dtype, r[k], g);
#pragma unroll
      for (int i = 0; i < kPer; ++i) q = fmaf(g[i], g[i], q);
      sum += (double)q;
    }
  }
  sum = sum_of_block(sum, shared);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}
__global__ void __launch_bounds__(1024) k_norm_join(const double* parts, uint32_t n, float grad_scale, float* norm) {
  __shared__ double shared[32];
  pdl_enter();
  double sum = 0.0;
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) sum += parts[i];
  sum = sum_of_block(sum, shared);
  if (threadIdx.x == 0) *norm = (float)(sqrt(sum) * fabs((double)grad_scale));
}

// ---- launching -----------------------------------------------------------------------------

// Blocks of values in a chunk, the work of a block of threads.  A step with 32-bit states has one for each warp: new blocks of threads keep more loads on their
// way than a loop does (100 M values: one 409 us, two 419, four 426; one vector of 11 M 67, 70, 73).  With 8 bits, where there is more to do before the
// first value (Philox's keys, the tensor), eight for each of four warps (314 us with two, 298 with four, 293), fewer where SMs would have none.
uint64_t blocks_of(const cvlc_adamw_tensor* t, uint32_t n) {
  uint64_t blocks = 0;
  for (uint32_t i = 0; i < n; ++i) blocks += (t[i].n + kPer + kBlock - 1) / kBlock;
  return blocks;
}
uint32_t step_chunk(uint64_t blocks, uint32_t bits) {
  uint32_t chunk = kWarps;
  while (bits == 8 && chunk < 4 * kWarps && blocks / (2 * chunk) >= 8 * kNumSM) chunk *= 2;
  return chunk;
}
// At most kNormChunks in all (500 M bf16 values: ten for each SM 188 us, 24 175, 64 183, 256 224): many, that blocks end together; not too many, since each has to find its tensor.
uint32_t norm_chunk(uint64_t blocks) {
  if (blocks < 8 * kWarps * (uint64_t)kNumSM) return kWarps;
  const uint64_t whole = 4 * kWarps, chunk = (blocks + kNormChunks - 1) / kNormChunks;
  return (uint32_t)((chunk + whole - 1) / whole * whole);
}
uint32_t misplaced(const void* p, size_t size, uint32_t per) { return (uint32_t)(reinterpret_cast<uintptr_t>(p) / size % per); }

TensorDesc describe(const cvlc_adamw_tensor& t, const StepScalars& s, uint32_t bits, bool norm) {
  auto bytes = [](uint32_t dtype) { return dtype == CVLC_F32 ? (size_t)4 : (size_t)2; };
  TensorDesc d = {};
  d.n = t.n, d.grad = t.grad_dev;
  const size_t size_g = bytes(s.grad_dtype);
  if (norm) {
    d.lead = (uint16_t)misplaced(t.grad_dev, size_g, kPer);
    d.vec = kVecGrad;
    return d;
  }
  d.param = t.param_dev, d.m = t.m_dev, d.v = t.v_dev, d.scale = reinterpret_cast<float2*>(t.scale_dev), d.copy = t.copy_dev;
  d.lr = t.lr, d.decay = t.weight_decay;
  const size_t size_p = bytes(s.param_dtype), size_s = bits == 8 ? 1 : 4;
  if (bits != 8) d.lead = (uint16_t)misplaced(t.param_dev, size_p, kPer);
  auto fits = [&](const void* p, size_t size, size_t vector) { return (reinterpret_cast<uintptr_t>(p) + vector * 64 - d.lead * size) % vector == 0; };
  d.vec = (fits(t.param_dev, size_p, 16) ? kVecParam : 0) | (fits(t.grad_dev, size_g, 16) ? kVecGrad : 0) |
          (fits(t.m_dev, size_s, bits == 8 ? 8 : 16) ? kVecM : 0) | (fits(t.v_dev, size_s, bits == 8 ? 8 : 16) ? kVecV : 0) |
          (fits(t.copy_dev, 2, 16) ? kVecCopy : 0);
  return d;
}

// Calls f with the descriptors of at most CAP tensors from `at` on; false behind the last one
template <uint32_t CAP, class F>
cudaError_t with_list(const cvlc_adamw_tensor* t, uint32_t n, const StepScalars& s, uint32_t bits, bool norm, uint32_t tensor0, F&& f) {
  TensorList<CAP> L;
  L.s = s;
  L.s.tensor0 = tensor0;
  L.n = 0, L.chunks = 0;
  for (uint32_t i = 0; i < n; ++i) {
    TensorDesc& d = L.t[L.n++];
    d = describe(t[i], s, bits, norm);
    d.first = L.chunks;
    const uint64_t blocks = (d.n + d.lead + kBlock - 1) / kBlock;
    L.chunks += (uint32_t)((blocks + s.chunk - 1) / s.chunk);
  }
  if (L.chunks == 0) return cudaSuccess;
  f(L);
  return cudaGetLastError();
}
template <class F>
cudaError_t by_lists(const cvlc_adamw_tensor* t, uint32_t n, const StepScalars& s, uint32_t bits, bool norm, F&& f) {
  for (uint32_t at = 0; at < n;) {
    const uint32_t left = n - at, now = left < kMany ? left : kMany;
    const cudaError_t e = now <= kFew    ? with_list<kFew>(t + at, now, s, bits, norm, at, f)
                          : now <= kSome ? with_list<kSome>(t + at, now, s, bits, norm, at, f)
                                         : with_list<kMany>(t + at, now, s, bits, norm, at, f);
    if (e != cudaSuccess) return e;
    at += now;
  }
  return cudaSuccess;
}
template <uint32_t CAP>
void run_step(const TensorList<CAP>& L, uint32_t bits, cudaStream_t st) {
  if (bits == 8) launch_kernel(kKAdamw, k_adamw<true, CAP>, dim3(L.chunks), dim3(kStepThreads<true>), 0, st, false, L);
  else launch_kernel(kKAdamw, k_adamw<false, CAP>, dim3(L.chunks), dim3(kStepThreads<false>), 0, st, false, L);
}

}  // namespace

cudaError_t launch_adamw(const cvlc_adamw_tensor* t, uint32_t n, const cvlc_adamw_args& a, cudaStream_t st) {
  StepScalars s = {};
  s.lr = (float)a.lr, s.b1 = (float)a.beta1, s.b1r = (float)(1.0 - a.beta1), s.b2 = (float)a.beta2, s.b2r = (float)(1.0 - a.beta2), s.eps = (float)a.eps;
  s.beta1 = a.beta1, s.beta2 = a.beta2;
  s.ic1 = (float)(1.0 / (1.0 - pow(a.beta1, (double)a.step))), s.ic2 = (float)(0x1p24 / (1.0 - pow(a.beta2, (double)a.step)));
  s.grad_scale = a.grad_scale, s.max_norm = a.max_norm, s.norm = a.norm_dev, s.lr_dev = a.lr_dev, s.step_dev = a.step_dev, s.seed = a.seed, s.step = a.step;
  s.param_dtype = a.param_dtype, s.grad_dtype = a.grad_dtype, s.copy_dtype = a.copy_dtype, s.status = a.status_dev;
  s.chunk = step_chunk(blocks_of(t, n), a.state_bits);
  return by_lists(t, n, s, a.state_bits, false, [&](const auto& L) { run_step(L, a.state_bits, st); });
}

size_t norm_ws_bytes(uint32_t n) { return align256(((size_t)kNormChunks + n) * sizeof(double)); }

cudaError_t launch_grad_norm(const cvlc_adamw_tensor* t, uint32_t n, uint32_t dtype, float grad_scale, float* norm, void* ws, cudaStream_t st) {
  StepScalars s = {};
  s.grad_dtype = dtype;
  s.chunk = norm_chunk(blocks_of(t, n));
  double* parts = static_cast<double*>(ws);
  uint32_t made = 0;
  const cudaError_t e = by_lists(t, n, s, 32, true, [&](const auto& L) {
    launch_kernel(kKNormParts, k_norm_parts<sizeof(L.t) / sizeof(L.t[0])>, dim3(L.chunks), dim3(kThreads), 0, st, false, L, parts + made);
    made += L.chunks;
  });
  if (e != cudaSuccess) return e;
  launch_kernel(kKNormJoin, k_norm_join, dim3(1), dim3(made > 256 ? 1024 : 256), 0, st, made != 0, parts, made, grad_scale, norm);
  return cudaGetLastError();
}

}  // namespace cvlc
