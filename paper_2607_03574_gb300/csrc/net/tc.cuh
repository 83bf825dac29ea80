// Tensor-core building blocks for sm_103a: tiles that the tensor memory accelerator (TMA) copies into shared
// memory in the 128-byte swizzle, products of them that accumulate in tensor memory (tcgen05), and the
// mbarriers between the two.  Every wait has a limit, after which the caller gives up.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace ndvm {
namespace tc {

__device__ __forceinline__ uint32_t smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// Waits for the phase of `parity` to end; false once `*stop` is set, or after kWaitNs, which sets it: the
// longest wait of a sound launch, for one tile's whole sum, is some milliseconds (seconds at the largest sizes that
// the C ABI takes).
constexpr uint64_t kWaitNs = 10000000000ull;
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile int* stop) {
  if (barrier_try(bar, parity)) return true;
  const uint64_t start = now_ns();
  while (!barrier_try(bar, parity)) {
    if (*stop) return false;
    if (now_ns() - start > kWaitNs) {
      *stop = 1;
      return false;
    }
  }
  return true;
}
// the same for what is in flight when a launch gives up
__device__ __forceinline__ void barrier_drain(uint32_t bar, uint32_t parity) {
  const uint64_t start = now_ns();
  while (!barrier_try(bar, parity) && now_ns() - start <= kWaitNs) {}
}

// The blocks of a launch work alone (kCtas = 1) or in pairs of a cluster (2), whose products one block issues
// for both: each holds its own rows of A and half of B's, and its own rows of the sums.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address, for the copies' and arrivals' use, of the first block's `p`
__device__ __forceinline__ uint32_t in_first(uint32_t p) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(p));
  return r;
}
__device__ __forceinline__ void barrier_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// One lane of a converged warp.  Copies, products and commits take their operands from registers that a warp shares; where the
// compiler sees that one lane of a whole warp issues them, it computes those there (otherwise it goes over the lanes of a
// divergent branch, operand by operand: a step of the products took 600 cycles more to issue than to run).
__device__ __forceinline__ bool elect() {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok));
  return ok != 0;
}
// asks for a tensor's map ahead of its first copy
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// a box of the tensor at (x, y) to shared memory; its bytes count on the barrier (which for a pair is in_first's)
template <int kCtas>
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (kCtas == 1)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (kCtas == 1)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(to), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// a box of shared memory to the tensor at (x, y[, z]); what lies outside it is left out
__device__ __forceinline__ void store_box(const CUtensorMap* map, int x, int y, uint32_t from) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(map), "r"(from), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap* map, int x, int y, int z, uint32_t from) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(from), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// until all but the last `kLeft` groups of this thread's stores have read their shared memory
template <int kLeft>
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory"); }
// makes this thread's writes to shared memory visible to the copies
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void store16(uint32_t to, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 32 rows of 32 16-bit elements in the 64-byte swizzle to rows that start anywhere, a row a warp and store, eight read at once
template <typename T>
__device__ __forceinline__ void unstage(const char* buffer, int lane, T* out, int64_t stride, int rows, int cols) {
  for (int r0 = 0; r0 < rows; r0 += 8) {
    T v[8];
#pragma unroll
    for (int u = 0; u < 8; u++) v[u] = *reinterpret_cast<const T*>(buffer + (r0 + u) * 64 + ((lane / 8 ^ ((r0 + u) >> 1 & 3)) << 4) + lane % 8 * 2);
#pragma unroll
    for (int u = 0; u < 8; u++)
      if (r0 + u < rows && lane < cols) out[(r0 + u) * stride + lane] = v[u];
  }
}

template <int kCtas, int kColumns>
__device__ __forceinline__ void tmem_alloc(uint32_t to) {
  if constexpr (kCtas == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int kCtas, int kColumns>
__device__ __forceinline__ void tmem_free(uint32_t addr) {
  if constexpr (kCtas == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(kColumns));
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(kColumns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D (+)= A B^T for 16 of the contraction: 16-bit operands in shared memory, binary32 sums in tensor memory
template <int kCtas>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  if constexpr (kCtas == 1)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}
// The same for 32 of the contraction of e4m3 operands in 8-bit blocks: a and b's scales (a byte of a column of tensor
// memory for each row, by the descriptor's scale ids) are powers of two.
template <int kCtas>
__device__ __forceinline__ void mma_blocks(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t a_scales, uint32_t b_scales, bool add) {
  if constexpr (kCtas == 1)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add) : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add) : "memory");
}
// 512 bytes of shared memory (32 lanes of 16 bytes) to 4 columns of tensor memory, the same for each quarter of the lanes; products
// issued later by this thread see them (a pair's blocks both copy, each its own)
template <int kCtas>
__device__ __forceinline__ void copy_scales(uint32_t to, uint32_t from) {
  // no swizzle, groups of 8 lanes 128 bytes apart
  const uint64_t desc = ((uint64_t)(from >> 4) & 0x3fff) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
  if constexpr (kCtas == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
}
// arrives on the barrier (of a pair: on both blocks') when the products issued so far are done
template <int kCtas>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (kCtas == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}

// 32 columns of this thread's lane of tensor memory
__device__ __forceinline__ void tmem_load32(float (&v)[32], uint32_t addr) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
#pragma unroll
  for (int i = 0; i < 32; i++) v[i] = __uint_as_float(r[i]);
}
// waits for the loads; what is done with their values comes after (they pass through)
__device__ __forceinline__ void tmem_loaded(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]),
                 "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]),
                 "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]),
                 "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
                 "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]),
                 "+f"(v[31])
               :: "memory");
}

// Shared-memory descriptor of an operand in the 128-byte swizzle.  Contraction contiguous: a line of 128
// bytes is 64 of the contraction, groups of 8 lines (rows or columns of the product) are 1024 bytes apart.
// Rows contiguous: a line is 64 rows, groups of 8 lines (of the contraction) are 1024 bytes apart, the next
// 64 rows start 8192 bytes on.
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool rows_contiguous) {
  const uint64_t leading = rows_contiguous ? 8192 >> 4 : 1, stride = 1024 >> 4;
  return ((uint64_t)(addr >> 4) & 0x3fff) | leading << 16 | stride << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor: binary32 sums, both operands half or both bfloat16, which of them have rows contiguous
__host__ __device__ constexpr uint32_t instruction(bool bf16, bool a_rows, bool b_rows, int m, int n) {
  return 1u << 4 | (uint32_t)bf16 << 7 | (uint32_t)bf16 << 10 | (uint32_t)a_rows << 15 | (uint32_t)b_rows << 16 |
         (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}
// and for e4m3 operands in 8-bit blocks; id: which byte of their columns the scales are
__host__ __device__ constexpr uint32_t instruction_blocks(int m, int n, int id) {
  return (uint32_t)id << 4 | (uint32_t)(n / 8) << 17 | 1u << 23 | (uint32_t)(m / 128) << 27 | (uint32_t)id << 29;
}

}  // namespace tc
}  // namespace ndvm
