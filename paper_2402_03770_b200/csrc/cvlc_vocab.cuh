// The two ends of a client's local step at which the vocabulary is, rows of logits (top logits, distillation) and rows of the
// embedding table (lookup, gradient), and the optimiser behind it.  What their kernels share: element types and 16-byte vectors of them.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>

#include <type_traits>

#include "cvlc_common.cuh"

namespace cvlc {

constexpr uint32_t kMaxClusterBlocks = 8;  // blocks of a cluster that every device takes

// ---- launchers (cvlc_logits.cu, cvlc_embed.cu) --------------------------------------------

struct TopArgs {
  const void* logits;
  uint64_t rows, row_stride;
  uint32_t vocab, k;
  float temperature;
  int32_t* ids;
  float* logp;
  float c2;                       // log2(e) / temperature
  float twice_it, twice_it_rest;  // 2 / temperature, in two numbers
};
cudaError_t launch_top_logits(const TopArgs& a, uint32_t dtype, cudaStream_t st);

struct DistillArgs {
  const void* logits;
  uint64_t rows, row_stride, grad_stride;
  uint32_t vocab, k, rest;
  float temperature;
  const int32_t* ids;
  const float* logp;
  const float* row_weight;  // or nullptr
  int32_t* status;          // or nullptr
  float* loss;              // the loss and the step write it
  float* stats;             // the loss writes it (or nullptr), the gradient reads it
  void* grad;               // the gradient and the step write it
  float c2;                 // log2(e) / temperature
};
enum DistillKind { kDistillLoss, kDistillGrad, kDistillStep };
cudaError_t launch_distill(const DistillArgs& a, uint32_t dtype, DistillKind kind, cudaStream_t st);
cudaError_t launch_selftest_ring(const float* row, uint32_t cuts, int give_back, uint64_t most, int32_t* status, float* seen, cudaStream_t st);

struct EmbedArgs {
  const void* table;
  uint64_t vocab, table_stride, n, out_stride;
  uint32_t dim, token_bytes;
  const void* tokens;
  float scale;
  void* out;
  int32_t* status;  // or nullptr
};
cudaError_t launch_embed(const EmbedArgs& a, uint32_t dtype, cudaStream_t st);

struct EmbedGradArgs {
  const void* tokens;
  const void* grad;
  uint64_t vocab, n, grad_stride, update_stride;
  uint32_t dim, token_bytes;
  float scale;
  float* update;
  int accumulate;
  void* ws;
};
cudaError_t launch_embed_grad(const EmbedGradArgs& a, uint32_t dtype, cudaStream_t st);
size_t embed_grad_ws_bytes(uint64_t n, uint32_t dim);

// A fault for the self-test, in one of a call's products: the tile of every block from which on it copies nothing, the one at which its readers give up, the limit of waits
struct HeadFault {
  uint32_t product, copy, tile;
  uint64_t most;
};
size_t head_ws_bytes(const cvlc_head& a, uint32_t pieces);
cudaError_t launch_head(const cvlc_head& a, uint32_t pieces, float* loss, void* d_hidden, uint64_t d_hidden_stride, void* d_head, uint64_t d_head_stride, void* ws,
                        cudaStream_t st, const HeadFault* fault = nullptr);  // pieces = 0: the loss alone

cudaError_t launch_adamw(const cvlc_adamw_tensor* tensors, uint32_t n, const cvlc_adamw_args& a, cudaStream_t st);
size_t norm_ws_bytes(uint32_t n);
cudaError_t launch_grad_norm(const cvlc_adamw_tensor* tensors, uint32_t n, uint32_t dtype, float grad_scale, float* norm, void* ws, cudaStream_t st);

#ifdef __CUDACC__

// ---- elements ------------------------------------------------------------------------------

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <class T>
constexpr int kPerVec = 16 / (int)sizeof(T);  // elements of a 16-byte vector

// 16 bytes of elements, widened and narrowed (one rounding to nearest)
template <class T>
__device__ __forceinline__ void widen(const uint4& raw, float (&v)[kPerVec<T>]);
template <>
__device__ __forceinline__ void widen<float>(const uint4& raw, float (&v)[4]) {
  v[0] = __uint_as_float(raw.x), v[1] = __uint_as_float(raw.y), v[2] = __uint_as_float(raw.z), v[3] = __uint_as_float(raw.w);
}
template <>
__device__ __forceinline__ void widen<__half>(const uint4& raw, float (&v)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __half2 h;
    memcpy(&h, &w[i], 4);
    const float2 f = __half22float2(h);
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}
template <>
__device__ __forceinline__ void widen<__nv_bfloat16>(const uint4& raw, float (&v)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
}
template <class T>
__device__ __forceinline__ uint4 narrow(const float (&v)[kPerVec<T>]);
template <>
__device__ __forceinline__ uint4 narrow<float>(const float (&v)[4]) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
template <>
__device__ __forceinline__ uint4 narrow<__half>(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    memcpy(&w[i], &h, 4);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <>
__device__ __forceinline__ uint4 narrow<__nv_bfloat16>(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    memcpy(&w[i], &h, 4);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// the elements of a vector whose bits are set, put to minus infinity
template <class T>
__device__ __forceinline__ uint32_t drop_of_word(uint32_t w, uint32_t bits) {
  if constexpr (sizeof(T) == 4) {
    return bits & 1 ? 0xFF800000u : w;
  } else {
    constexpr uint32_t inf = std::is_same<T, __half>::value ? 0xFC00u : 0xFF80u;
    if (bits & 1) w = (w & 0xFFFF0000u) | inf;
    if (bits & 2) w = (w & 0xFFFFu) | (inf << 16);
    return w;
  }
}
template <class T>
__device__ __forceinline__ void drop_elements(uint4& raw, uint32_t bits) {
  constexpr int per = 4 / (int)sizeof(T);
  raw.x = drop_of_word<T>(raw.x, bits);
  raw.y = drop_of_word<T>(raw.y, bits >> per);
  raw.z = drop_of_word<T>(raw.z, bits >> (2 * per));
  raw.w = drop_of_word<T>(raw.w, bits >> (3 * per));
}

// 2^x, relative error below 2^-22; 2^-inf = 0
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

#endif  // __CUDACC__

}  // namespace cvlc
