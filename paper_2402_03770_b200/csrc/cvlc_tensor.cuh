// What a kernel needs to feed the tensor cores of sm_100a: barriers in shared memory with bounded waits, tile copies by tensor maps, descriptors of
// operands in shared memory, products into tensor memory and reading them back.
#pragma once

#include <cuda.h>

#include "cvlc_common.cuh"

namespace cvlc {

// A matrix of 16-bit elements, `rows` rows of `cols` (contiguous), `stride` elements apart, read in tiles of box_cols x box_rows with the swizzle of 128 bytes;
// what lies outside reads as 0.  Its base lies on 16 bytes and the stride is a multiple of 8 elements.
bool make_tensor_map(CUtensorMap* map, const void* base, bool bf16, uint64_t cols, uint64_t rows, uint64_t stride, uint32_t box_cols, uint32_t box_rows);

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// Two blocks of a cluster (CG = 2) make a tile of twice the rows together: each copies its half of both operands, the first one, the leader, issues the
// products of both, and what the leader waits for is reported to its barriers.  The same place in the leader's shared memory:
template <int CG>
__device__ __forceinline__ uint32_t leader_at(uint32_t at) {
  if constexpr (CG == 1) return at;
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(at));
  return r;
}
template <int CG>
__device__ __forceinline__ uint32_t pair_rank() {
  if constexpr (CG == 1) return 0;
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
template <int CG>
__device__ __forceinline__ void pair_sync() {  // of all threads
  if constexpr (CG == 1) __syncthreads();
  else asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A word in the shared memory of a pair's other block
__device__ __forceinline__ uint32_t other_at(uint32_t at) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(pair_rank<2>() ^ 1));
  return r;
}
__device__ __forceinline__ void shared_store(uint32_t at, uint32_t x) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(x) : "memory"); }
__device__ __forceinline__ uint32_t shared_load(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}

__device__ __forceinline__ void mbar_init(uint64_t* b, uint32_t n) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(smem_at(b)), "r"(n)); }
__device__ __forceinline__ void mbar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(smem_at(b)), "r"(bytes) : "memory");
}
// bytes that are expected and will not come count as come
__device__ __forceinline__ void mbar_came(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_at(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* b) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(smem_at(b)) : "memory"); }
// The tensor memory has been read (tensor_loaded() has waited for it), and nothing else is handed over: an arrival that released would wait for the stores of all that
// the thread has written (4096 x 256 x 50048, the logits' statistics: 137 -> 119 us).
template <int CG>
__device__ __forceinline__ void mbar_arrive_leader(uint64_t* b) {
  if constexpr (CG == 1) mbar_arrive(b);
  else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_at<CG>(smem_at(b))) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint64_t* b, uint32_t parity) {
  uint32_t done;
  // suspended for up to 10 ms: threads that ask again and again take from those that work (a product of 4096 x 2048 x 50048: 604 -> 559 us)
  asm volatile("{.reg .pred p;\n mbarrier.try_wait.parity.shared.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;}"
               : "=r"(done)
               : "r"(smem_at(b)), "r"(parity), "r"(10000000u)
               : "memory");
  return done != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Waits are bounded: `late` (in shared memory, 0 at first) is set by the first that runs out, and ends the others.
constexpr uint64_t kMostWait = 4000000000ull;  // nanoseconds
__device__ __forceinline__ bool mbar_wait(uint64_t* b, uint32_t parity, uint32_t* late, uint64_t most = kMostWait) {
  if (mbar_try(b, parity)) return true;
  const uint64_t began = now_ns();
  for (;;) {
    if (mbar_try(b, parity)) return true;
    if (*static_cast<volatile uint32_t*>(late)) return false;
    if (now_ns() - began > most) {
      *static_cast<volatile uint32_t*>(late) = 1;
      return false;
    }
  }
}

// ---- copies --------------------------------------------------------------------------------
// `bar`: the leader's
template <int CG>
__device__ __forceinline__ void load_tile(const CUtensorMap& map, uint32_t to, uint32_t bar, uint32_t x, uint32_t y) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to),
                 "l"(&map), "r"(bar), "r"(x), "r"(y)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to), "l"(&map), "r"(bar),
                 "r"(x), "r"(y)
                 : "memory");
}

// A box of 64 columns by 32 rows that a warp has left in shared memory (swizzled, on 1024 bytes) to where the map says; what lies outside is left out.  By one
// thread, behind shared_written() of all; the buffer is free again behind tiles_read(), the copy made behind tiles_stored().
__device__ __forceinline__ void shared_written() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void store_tile(const CUtensorMap& map, uint32_t from, uint32_t x, uint32_t y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n cp.async.bulk.commit_group;" ::"l"(&map), "r"(from), "r"(x),
               "r"(y)
               : "memory");
}
__device__ __forceinline__ void tiles_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tiles_stored() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ---- operands ------------------------------------------------------------------------------
// Both kinds of tile hold lines of 128 bytes, eight of which are one swizzled group of 1024.
//   along the sum ("K first"): a line is 64 values of the sum of one row; groups of eight rows follow one another.  16 values of the sum
//   further: 32 bytes.
//   along the rows ("rows first"): a line is 64 rows of one value of the sum; groups of eight values of the sum follow one another, 64 further rows are a
//   tile of their own behind all values of the sum.  16 values of the sum further: 2048 bytes.
// `values`: of the sum, in a tile of rows first
template <bool ROWS_FIRST>
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t values) {
  const uint64_t leading = ROWS_FIRST ? values * 128 >> 4 : 1;
  constexpr uint64_t stride = 1024 >> 4;
  return (uint64_t)((at & 0x3FFFF) >> 4) | leading << 16 | stride << 32 | 1ull << 46 | 2ull << 61;
}
template <bool ROWS_FIRST>
constexpr uint32_t kStepBytes = ROWS_FIRST ? 2048 : 32;

// products of bf16 or fp16 (not mixed), sums in fp32, m x n at a time
__host__ __device__ constexpr uint32_t product_kind(bool bf16, bool a_rows_first, bool b_rows_first, uint32_t m, uint32_t n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_rows_first ? 1u << 15 : 0u) | (b_rows_first ? 1u << 16 : 0u) | (n >> 3) << 17 | (m >> 4) << 24;
}
template <int CG>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
  if constexpr (CG == 2)
    asm volatile("{.reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;}" ::"r"(d), "l"(a), "l"(b), "r"(kind),
                 "r"((uint32_t)add)
                 : "memory");
  else
    asm volatile("{.reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;}" ::"r"(d), "l"(a), "l"(b), "r"(kind),
                 "r"((uint32_t)add)
                 : "memory");
}
// arrives at the barrier (of both blocks of a pair) when the products so far are complete
template <int CG>
__device__ __forceinline__ void commit(uint64_t* b) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_at(b)), "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(b)) : "memory");
}
template <int CG>
__device__ __forceinline__ void tensor_alloc(uint32_t* at) {  // all of the SM's tensor memory, by one warp
  if constexpr (CG == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <int CG>
__device__ __forceinline__ void tensor_free(uint32_t at) {
  if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at));
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(at));
}
__device__ __forceinline__ void tensor_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of this thread's row; the values are there after tensor_loaded()
__device__ __forceinline__ void tensor_load(uint32_t at, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
      "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
        "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]),
        "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(at));
}
// (they pass through it, so that nothing is made of them before)
__device__ __forceinline__ void tensor_loaded(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]),
                 "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]),
                 "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]),
                 "+f"(v[31])
               :
               : "memory");
}

// 32 bytes, a whole sector, to a place on 32 bytes
__device__ __forceinline__ void store_sector(void* at, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
               "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void load_sector(const void* at, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(at));
}

#endif  // __CUDACC__

}  // namespace cvlc
