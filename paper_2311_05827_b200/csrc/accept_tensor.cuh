// Tensor-core building blocks (sm_100a): tile loads through tensor maps, tensor memory, and the matrix instruction for
// 8-bit operands with block scales.  Every wait on a barrier is bounded (mbarrier_wait).
#pragma once
#include <cuda.h>

#include "accept_async.cuh"

namespace accept {

// One lane of the warp, always the same.  The warp runs its loop as a whole and one lane issues: what is the same for the
// whole warp can then stay in uniform registers, where the matrix instructions take their descriptors from.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// mbarrier_wait by a whole warp, with one result for all lanes; gives up after `limit_ns`.
__device__ __forceinline__ bool mbarrier_wait_warp(uint32_t bar, uint32_t parity, unsigned long long limit_ns = kCopyWaitNs) {
  unsigned long long t0 = 0;
  for (uint32_t it = 0;; ++it) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (__all_sync(0xffffffffu, done)) return true;
    if ((it & 63u) == 63u) {
      unsigned long long now;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (t0 == 0) t0 = now;
      else if (__any_sync(0xffffffffu, now - t0 > limit_ns)) return false;
    }
  }
}

// One box of a tensor map into shared memory; the barrier counts its bytes.  Boxes past the tensor's end are filled
// with zeros (and counted in full).
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---- tensor memory: 128 lanes x 512 columns of 32 bits for each SM ----
__device__ __forceinline__ void tensor_alloc(uint32_t result, uint32_t columns) {  // one whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tensor_free(uint32_t address, uint32_t columns) {  // the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: thread l gets row l.
__device__ __forceinline__ void tensor_read(uint32_t address, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
        "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
        "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(address));
}
__device__ __forceinline__ void tensor_read(uint32_t address, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(address));
}
__device__ __forceinline__ void tensor_read_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- descriptors of operands in shared memory ----
// Bits 0-13 address / 16, 32-45 stride between groups of eight rows / 16, 46-48 = 1, 61-63 swizzle.
// Operand tiles: rows of 128 bytes, groups of eight rows 1024 bytes apart, 128-byte swizzle (2).
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t address) {
  return (uint64_t)(address >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Scales: 32 rows of 16 bytes, groups of eight rows 128 bytes apart, no swizzle.
__device__ __forceinline__ uint64_t scale_descriptor(uint32_t address) {
  return (uint64_t)(address >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}
// 512 bytes of scales (128 rows x four blocks) to four columns, repeated for the four lane groups.
__device__ __forceinline__ void scale_copy(uint32_t tensor, uint64_t descriptor) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tensor), "l"(descriptor) : "memory");
}

// Instruction descriptor for 8-bit operands with scales: formats at bits 7 and 10 (E4M3 0, E5M2 1), N / 8 at 17,
// scales that are powers of two (23), M / 16 at 24, which byte of the four in a scale word at 4 (B) and 29 (A).
__host__ __device__ constexpr uint32_t scaled_instruction(uint32_t format_a, uint32_t format_b, uint32_t m, uint32_t n) {
  return (format_a << 7) | (format_b << 10) | ((n >> 3) << 17) | (1u << 23) | ((m >> 4) << 24);
}
__device__ __forceinline__ uint32_t with_scale_byte(uint32_t instruction, uint32_t byte) { return instruction | (byte << 4) | (byte << 29); }

// d (+)= a b^T over 32 values of k: one thread issues it for the block.
__device__ __forceinline__ void scaled_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t scale_a, uint32_t scale_b, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(instruction), "r"(scale_a), "r"(scale_b), "r"((uint32_t)add) : "memory");
}
// The barrier is arrived at once all matrix instructions issued so far by this thread are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- pairs of blocks (cta_group::2): two SMs work on one tile, the even block of the pair issues ----
// A box into this block's shared memory whose bytes the given barrier counts: an address in the cluster, of either block.
__device__ __forceinline__ void pair_tile_load(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t cluster_bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void pair_tensor_alloc(uint32_t result, uint32_t columns) {  // one whole warp of each block
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void pair_tensor_free(uint32_t address, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}
// Each block's scales, at the same place in both, to its own tensor memory.
__device__ __forceinline__ void pair_scale_copy(uint32_t tensor, uint64_t descriptor) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tensor), "l"(descriptor) : "memory");
}
// 256 rows of a (128 in each block's shared memory) by the rows of b (half in each).
__device__ __forceinline__ void pair_scaled_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t scale_a, uint32_t scale_b, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(instruction), "r"(scale_a), "r"(scale_b), "r"((uint32_t)add) : "memory");
}
// The barrier at this place in both blocks is arrived at once the matrix instructions issued so far are done.
__device__ __forceinline__ void pair_mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mbarrier_arrive_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

// ---- tile stores ----
__device__ __forceinline__ void tile_store(const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void tile_add(const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t src) {  // fp32, added where the tile lies
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING>  // all but the last PENDING groups have been read: their sources may be reused
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ void store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }            // written
__device__ __forceinline__ void shared_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- clusters ----
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t address_in(uint32_t shared_address, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(shared_address), "r"(rank));
  return r;
}
__device__ __forceinline__ float ld_cluster_one(uint32_t address) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(address) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_cluster(uint32_t address) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(address) : "memory");
  return v;
}

}  // namespace accept
