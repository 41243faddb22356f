// Fifth-generation tensor cores, tensor copies and barriers in shared memory: thin wrappers of the PTX
// instructions that the kernels use, and bounded waits.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace efcp {
namespace tc {

__device__ __forceinline__ uint32_t smem_of(const void* p) {
  return uint32_t(__cvta_generic_to_shared(p));
}

// ------------------------------------------------------------------ barriers
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ bool bar_poll(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
__device__ __forceinline__ uint64_t clock_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

constexpr uint64_t kWaitNs = 2000000000ull;  // limit of a wait: 2 s
constexpr uint64_t kDrainNs = 500000000ull;  // and of the waits for what is in flight after one ran out

// Waits for the barrier's phase; false when the limit passes or another thread of the block has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up,
                                         uint64_t limit = kWaitNs) {
  for (int i = 0; i < 64; ++i)
    if (bar_poll(bar, parity)) return true;
  const uint64_t start = clock_ns();
  while (true) {
    for (int i = 0; i < 64; ++i)
      if (bar_poll(bar, parity)) return true;
    if (limit == kWaitNs && *gave_up) return false;
    if (clock_ns() - start > limit) {
      *gave_up = 1;
      return false;
    }
  }
}

// Waits for a counter in shared memory that another warp of the block moves on; false as above.
__device__ __forceinline__ bool count_wait(const volatile unsigned* counter, unsigned least, volatile int* gave_up) {
  const uint64_t start = clock_ns();
  while (int(*counter - least) < 0) {
    if (*gave_up) return false;
    if (clock_ns() - start > kWaitNs) {
      *gave_up = 1;
      return false;
    }
    __nanosleep(64);
  }
  __threadfence_block();
  return true;
}

// ------------------------------------------------------------------ pairs of blocks
__device__ __forceinline__ uint32_t pair_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of the first block's copy of something in shared memory.
__device__ __forceinline__ uint32_t of_first(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
// (What is told is that tensor memory was read, which the fence before it orders; a release for the whole cluster
// would wait for every store to global memory under way.)
__device__ __forceinline__ void bar_arrive_pair(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// What this thread wrote to shared memory comes before, for a thread that sees the phase done by bar_acquire_pair.  (A fence for
// the whole cluster in its place takes as long as two steps of a product.)
__device__ __forceinline__ void bar_release_pair(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_acquire_pair(uint32_t bar, uint32_t parity) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n"
      "}\n" ::"r"(bar),
      "r"(parity)
      : "memory");
}

// ------------------------------------------------------------------ tensor copies
// One box of a three-dimensional map into this block's shared memory, counted on a barrier of the pair's first
// block; the innermost coordinate is a multiple of 16 bytes.
__device__ __forceinline__ void load_box(const CUtensorMap* map, uint32_t dst, uint32_t bar, int x,
                                         int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
      "[%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// A box out of shared memory: stored, or added to what is there (fp32).
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
               "r"(src), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void add_box(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   map),
               "r"(src), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void close_stores() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// all but the newest LEFT groups of this thread have left shared memory
template <int LEFT>
__device__ __forceinline__ void stores_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// what was written to shared memory comes before copies out of it
__device__ __forceinline__ void fence_copies() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ------------------------------------------------------------------ tensor memory and products, of both blocks of a pair
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where),
               "r"(columns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}

// Descriptor of an operand in shared memory whose 64-element rows of 128 bytes are swizzled (128-byte mode).
//   inner dimension K:   eight rows of the outer dimension are 1024 bytes; groups of them lie side by side.
//   inner dimension M/N: eight rows of K are 1024 bytes, groups of them side by side; the next 64 of M/N lie
//                        8 KB further (64 rows of K).
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
  uint64_t d = (addr & 0x3FFFF) >> 4;
  d |= uint64_t(8192 >> 4) << 16;
  d |= uint64_t(1024 >> 4) << 32;
  d |= uint64_t(1) << 46;  // version of the format
  d |= uint64_t(2) << 61;  // 128-byte swizzle
  return d;
}

// fp32 accumulators; both operands fp16 or both bf16; M x N; which operands have M or N as their inner dimension
__host__ __device__ constexpr uint32_t instruction(bool bf16, int m, int n, bool a_mn, bool b_mn) {
  return (1u << 4) | (uint32_t(bf16) << 7) | (uint32_t(bf16) << 10) | (uint32_t(a_mn) << 15) |
         (uint32_t(b_mn) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}

// Issued by one thread of the first block: 256 rows, 128 of them in each block's tensor memory; each block holds its
// rows of A and half of the columns of B.
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t ins, bool add) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(ins), "r"(uint32_t(add))
      : "memory");
}
// Both blocks' barriers at this address are arrived at when all products issued so far by this thread are done.
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          bar),
      "h"(uint16_t(3))
      : "memory");
}

// 32 columns of this warp's 32 lanes, on their way until tmem_wait
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
// v has arrived, with every other load before it.  (It passes through, so that nothing reads it earlier.)
__device__ __forceinline__ void tmem_wait(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]),
                 "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]),
                 "+f"(v[14]), "+f"(v[15])
               :
               : "memory");
  asm volatile("" : "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                    "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]),
                    "+f"(v[30]), "+f"(v[31]));
}

}  // namespace tc
}  // namespace efcp
