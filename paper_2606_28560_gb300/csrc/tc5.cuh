// tc5.cuh -- PTX wrappers of the fifth-generation tensor core for kernels that
// run as pairs of CTAs (clusters of two, cta_group::2): TMEM, descriptors,
// MMA issue, cluster barriers, TMA.
#pragma once
#include "mma_common.cuh"

namespace fibattn {
namespace tc5 {

using mma::smem_u32;

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
// The address, in the cluster's shared window, of the same offset in CTA `rank`.
__device__ __forceinline__ unsigned map_to(unsigned addr, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ bool elect_one() {
    unsigned p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
    return p != 0;
}

// Bounded wait as mma::mbar_wait, with the acquire at cluster scope.
__device__ __forceinline__ bool wait_parity(unsigned bar, unsigned parity) {
    unsigned long long t0 = 0;
    for (unsigned it = 0;; ++it) {
        unsigned done;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                     " selp.u32 %0, 1, 0, p;\n}\n" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if ((it & 63u) == 0u) {
            const unsigned long long now = mma::global_ns();
            if (it == 0) t0 = now;
            else if (now - t0 > mma::kWaitLimitNs) return false;
        }
    }
}
__device__ __forceinline__ void init_barrier(unsigned bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void expect_bytes(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" :: "r"(bar), "r"(bytes) : "memory");
}
// bar: a cluster-window address.  Relaxed: what it hands over is TMEM, ordered
// by fence_before / fence_after; a release at cluster scope would wait for
// every global access of the thread as well.
__device__ __forceinline__ void arrive_cluster(unsigned bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" :: "r"(bar) : "memory");
}

// L2 policies of the copies: data that is read again and again (evict last) or
// passes through once (evict first).
__device__ __forceinline__ unsigned long long policy_keep() {
    unsigned long long p;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;\n" : "=l"(p));
    return p;
}
__device__ __forceinline__ unsigned long long policy_normal() {
    unsigned long long p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;\n" : "=l"(p));
    return p;
}
__device__ __forceinline__ unsigned long long policy_pass() {
    unsigned long long p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;\n" : "=l"(p));
    return p;
}

// TMA load of a box into this CTA's shared memory; its bytes are counted by a
// barrier of either CTA of the pair (cluster-window address).
__device__ __forceinline__ void load_box(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar,
                                         unsigned long long policy) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%2, %3, %4}], [%5], %6;\n"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap* map, unsigned src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];\n"
                 :: "l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
template <int N> __device__ __forceinline__ void store_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;\n" :: "n"(N) : "memory");
}
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];\n" :: "l"(map) : "memory");
}

// All 512 columns of both CTAs' TMEM; the base address goes to shared memory.
__device__ __forceinline__ void tmem_alloc(unsigned dst) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n" :: "r"(dst) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n");
}
__device__ __forceinline__ void tmem_free(unsigned base) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;\n" :: "r"(base));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }

// 32 consecutive columns of this warp's 32 lanes: r[j] is column j of the
// thread's lane (valid after tmem_wait_loads).
__device__ __forceinline__ void tmem_load32(unsigned addr, float* r) {
    unsigned* u = reinterpret_cast<unsigned*>(r);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
                   "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]),
                   "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]),
                   "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }

// Shared-memory matrix descriptor of a 128-byte-swizzled operand (version 1;
// offsets in units of 16 bytes).  Depth-major ("K-major", rows of 64 values of
// depth): stride = 1024 bytes between groups of eight rows.  Row-major
// ("MN-major", lines of 64 rows, one line per value of depth): stride = 1024
// bytes between groups of eight lines, lead = bytes between blocks of 64 rows.
__device__ __forceinline__ unsigned long long descriptor(unsigned addr, unsigned lead_bytes) {
    return (unsigned long long)((addr & 0x3ffffu) >> 4) | ((unsigned long long)(lead_bytes >> 4) << 16) |
           (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: bf16 x bf16 -> fp32, M = 256 rows over the pair, n columns.
__device__ __forceinline__ unsigned instruction(int n, bool a_row_major, bool b_row_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_row_major ? 1u : 0u) << 15) | ((b_row_major ? 1u : 0u) << 16) |
           ((unsigned)(n >> 3) << 17) | (16u << 24);
}
// One thread of the even CTA issues for the pair.
__device__ __forceinline__ void multiply(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory");
}
// Both CTAs' barrier at this offset gets one arrival once all MMAs issued so
// far by this thread are done.
__device__ __forceinline__ void commit_pair(unsigned bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n"
                 :: "r"(bar), "h"((unsigned short)3) : "memory");
}
template <int R> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" :: "n"(R)); }
template <int R> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" :: "n"(R)); }

}  // namespace tc5
}  // namespace fibattn
