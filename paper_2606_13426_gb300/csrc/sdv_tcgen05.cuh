// sdv_tcgen05.cuh - the fifth-generation matrix unit: tensor memory, operand descriptors, barriers.
#pragma once

#include <cstdint>

#include "sdv_tokens.cuh"

namespace sdv {

// ---- mbarriers.  Every wait gives up after kWaitMost clocks (two seconds), upon which the kernel ends with an error.
constexpr long long kWaitMost = 4000000000ll;
constexpr uint32_t kWaitHint = 1000000;           // nanoseconds that a waiting warp may sleep

__device__ __forceinline__ void barrier_init(uint64_t* bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint64_t* bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{ .reg .pred p;\n  mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2, %3;\n  selp.b32 %0, 1, 0, p; }"
      : "=r"(done)
      : "r"(smem_addr(bar)), "r"(parity), "r"(kWaitHint)
      : "memory");
  return done;
}
// Waits for the phase of that parity; false if it gave up, or another thread did (*dead).
__device__ __forceinline__ bool barrier_wait(uint64_t* bar, uint32_t parity, volatile int* dead) {
  if (barrier_try(bar, parity)) return true;
  const long long since = clock64();
#pragma unroll 1
  do {
    if (barrier_try(bar, parity)) return true;
    if (*dead) return false;
  } while (clock64() - since < kWaitMost);
  *dead = 1;
  return false;
}
// What this thread wrote to shared memory is there for the matrix unit.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- copies of whole vectors of 16 bytes from global to shared memory, which the barrier counts
__device__ __forceinline__ void barrier_expect(uint64_t* bar, uint32_t bytes) {   // an arrival that waits for them
  asm volatile("mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_bulk(uint32_t to, const void* from, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes),
               "r"(smem_addr(bar))
               : "memory");
}

// ---- tensor memory: 128 lanes of 512 columns of 32 bits
__device__ __forceinline__ void tmem_alloc(uint32_t* to, int columns) {          // by one warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, int columns) {            // by the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// The largest of three.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

#define SDV_R4(x, i) x(i), x(i + 1), x(i + 2), x(i + 3)
#define SDV_R16(x, i) SDV_R4(x, i), SDV_R4(x, i + 4), SDV_R4(x, i + 8), SDV_R4(x, i + 12)
#define SDV_R32(x) SDV_R16(x, 0), SDV_R16(x, 16)
// 32 columns of this thread's lane (a warp has the lanes 32 (warp % 4) on).  The registers are there after tmem_loaded.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t* r) {
#define SDV_OUT(i) "=r"(r[i])
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : SDV_R32(SDV_OUT)
      : "r"(at));
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : SDV_R16(SDV_OUT, 0)
      : "r"(at));
#undef SDV_OUT
}
// (The registers pass through, so that nothing that uses them comes before.)
__device__ __forceinline__ void tmem_loaded(uint32_t* r) {
#define SDV_INOUT(i) "+r"(r[i])
  asm volatile("tcgen05.wait::ld.sync.aligned;" : SDV_R32(SDV_INOUT)::"memory");
}
__device__ __forceinline__ void tmem_loaded16(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : SDV_R16(SDV_INOUT, 0)::"memory");
#undef SDV_INOUT
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* r) {
#define SDV_IN(i) "r"(r[i])
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
      SDV_R16(SDV_IN, 0)
      : "memory");
#undef SDV_IN
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- operands.  A tile in shared memory is [rows][64 elements of 16 bits], 128 bytes a row, whose eight pieces of 16 bytes
// are swizzled by the row: piece p of row r stands in place p ^ (r % 8).  Tiles start on 1024 bytes.
__device__ __forceinline__ uint32_t swizzled(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }
// The descriptor of such a tile, K along the row: start, 1024 bytes from eight rows to the next eight, 128-byte swizzle.
__device__ __forceinline__ uint64_t tile_desc(uint32_t at) {
  return (uint64_t)(at >> 4 & 0x3fff) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// The instruction's descriptor: fp32 sums of f16 products, both operands K-major.
__host__ __device__ constexpr uint32_t mma_desc(int m, int n) { return 1u << 4 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24; }
// One lane of a warp whose lanes are all here.
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{ .reg .pred p;\n  elect.sync _|p, 0xffffffff;\n  selp.b32 %0, 1, 0, p; }" : "=r"(yes));
  return yes;
}
// d (tensor memory) = a b' (+ d): 16 of K; a in shared memory, or in tensor memory.  By one thread.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  asm volatile("{ .reg .pred p;\n  setp.ne.b32 p, %4, 0;\n  tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a),
               "l"(b), "r"(desc), "r"((uint32_t)add)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add) {
  asm volatile("{ .reg .pred p;\n  setp.ne.b32 p, %4, 0;\n  tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a),
               "l"(b), "r"(desc), "r"((uint32_t)add)
               : "memory");
}
// Registers of a thread of this warp's four, from here on (sums over the block's warps stay within its launch).
template <int kN>
__device__ __forceinline__ void registers_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kN));
}
template <int kN>
__device__ __forceinline__ void registers_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kN));
}
// The barrier gets an arrival when all that this thread has issued before is done.
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

}  // namespace sdv
