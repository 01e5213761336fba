// Thin wrappers of the sm_100a instructions that the routed products use: tensor-map copies into shared memory, matrix
// instructions on tensor memory, and the waits between them (every one bounded).
#pragma once
#include <cuda.h>

#include "gm_common.cuh"

namespace gm {

// Kernels of the routed products are launched while the one before them in the stream still runs (programmatic dependent launch):
// what they do before grid_wait() touches no global memory, and behind it all that was queued before is done.
__device__ __forceinline__ void grid_launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Polls of a barrier before a wait gives up: a failed try_wait has itself waited for 1.5 us, so this is six seconds, far above any wait for a
// stage, its copies or a buffer of sums (microseconds).
constexpr int kT5SpinLimit = 1 << 22;

// Without back-off: these barriers hand over within a microsecond.
__device__ __forceinline__ bool t5_wait(u64* bar, u32 parity) {
  for (int i = 0; i < kT5SpinLimit; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return false;
}
// For the end of a sum, which lasts as long as its stages (0.2 to 0.5 us each: a sum over 2^30 values or places takes seconds), the limit grows
// with them: another one for each kT5StagesPerLimit.
constexpr u32 kT5StagesPerLimit = 1 << 20;
static_assert(kT5SpinLimit >= 2 * kT5StagesPerLimit, "twice the time of that many stages if they took a microsecond each, and a poll no more");
__device__ __forceinline__ bool t5_wait_sum(u64* bar, u32 parity, u32 stages) {
  for (u32 i = 0; i <= stages / kT5StagesPerLimit; ++i)
    if (t5_wait(bar, parity)) return true;
  return false;
}
// ---- pairs of blocks (clusters of two): the even one leads, its thread issues the matrix instructions for both
__device__ __forceinline__ u32 cluster_rank() {
  u32 r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of the leader's barrier that lies where `bar` does in this block
__device__ __forceinline__ u32 leader_bar(const u64* bar) {
  u32 a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(bar)));
  return a;
}
__device__ __forceinline__ void mbar_arrive_at(u32 cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Copies by tensor map into this block's memory; the bytes are announced on (and counted by) the leader's barrier.
__device__ __forceinline__ void mbar_arrive(u64* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_2d(u32 dst, const CUtensorMap* map, int x, int y, u32 bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_3d(u32 dst, const CUtensorMap* map, int x, int y, int z, u32 bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}

// From this block's memory into a result, by tensor map: what lies outside is not written.  One thread; the memory may be written again after
// tma_store_read(), and the block leave after tma_store_done().
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, u32 src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];\n\tcp.async.bulk.commit_group;" ::"l"(map), "r"(x), "r"(y), "r"(z),
               "r"(src)
               : "memory");
}
template <int kLeft> __device__ __forceinline__ void tma_store_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory"); }
__device__ __forceinline__ void tma_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// 16 bytes by the thread itself, of which the first `bytes` (0 .. 16) are read and the others become zero
__device__ __forceinline__ void copy16(u32 dst, const void* src, u32 bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(u32 dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// arrives on `bar` (of this block; initialised with one arrival per thread) when this thread's copies so far are there
__device__ __forceinline__ void copy_arrive(u64* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
__device__ __forceinline__ void copy_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// what this thread has seen written to shared memory is seen by the matrix instructions behind a barrier that it arrives on next
__device__ __forceinline__ void fence_to_matrix() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Tensor memory: a warp of each block of the pair allocates and frees.
__device__ __forceinline__ void tmem_alloc(u32* where, u32 columns) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(u32 addr, u32 columns) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void t5_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void t5_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// arrives on `bar` of both blocks when the matrix instructions issued so far by this thread are done
__device__ __forceinline__ void t5_commit(u64* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"(static_cast<uint16_t>(3))
               : "memory");
}
// 32 columns of this warp's 32 lanes: v[j] = lane's value in column addr + j.  t5_wait_ld() before the values are used.
__device__ __forceinline__ void t5_ld32(u32 (&v)[32], u32 addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
        "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]),
        "=r"(v[30]), "=r"(v[31])
      : "r"(addr));
}
__device__ __forceinline__ void t5_ld16(u32 (&v)[16], u32 addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                 "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
               : "r"(addr));
}
// Loaded values are used behind the wait: it "changes" them, so that no use can be moved in front of it.
__device__ __forceinline__ void t5_wait_ld16(u32 (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :
               : "memory");
}
// two products and sums in one instruction: acc += a * b, either half
__device__ __forceinline__ void fma2(u64& acc, u64 a, u64 b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b)); }
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 pair_of(u32 lo, u32 hi) {
  u64 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ void t5_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Descriptor of an operand in shared memory, 128-byte swizzle, the reduction along the 128-byte rows ("K-major"):
// groups of 8 rows lie 1024 bytes apart.
__device__ __forceinline__ u64 t5_desc_k(u32 addr) {
  return (static_cast<u64>(2) << 61) | (static_cast<u64>(1) << 46) | (static_cast<u64>(1024 >> 4) << 32) | (static_cast<u64>(1) << 16) | ((addr & 0x3ffff) >> 4);
}
// The same with the reduction across the rows ("MN-major"): 64 values of the operand's own dimension in a 128-byte row, 8 steps
// of the reduction in 1024 bytes, the next 64 values `block` bytes on.
__device__ __forceinline__ u64 t5_desc_mn(u32 addr, u32 block) {
  return (static_cast<u64>(2) << 61) | (static_cast<u64>(1) << 46) | (static_cast<u64>(1024 >> 4) << 32) | (static_cast<u64>(block >> 4) << 16) | ((addr & 0x3ffff) >> 4);
}
// Instruction descriptor: 32-bit sums; type 0 / 1 of both operands (f16 / bf16, or e4m3 / e5m2), MN-major flags, sizes.
__device__ __forceinline__ u32 t5_idesc(u32 type, bool a_mn, bool b_mn, u32 m, u32 n) {
  return (1u << 4) | (type << 7) | (type << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((n >> 3) << 17) | ((m >> 4) << 24);
}
__device__ __forceinline__ void t5_mma_f16(u32 d, u64 a, u64 b, u32 idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u)
      : "memory");
}
__device__ __forceinline__ void t5_mma_f8(u32 d, u64 a, u64 b, u32 idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u)
      : "memory");
}

}  // namespace gm
