// Cluster, distributed-shared-memory, dependent-launch and CTA-pair (cta_group::2) wrappers shared by the
// decode-shaped kernels.
#pragma once
#include "sm100_ptx.cuh"

namespace marlaas {
namespace sm100 {

__device__ __forceinline__ uint32_t dk_cluster_ctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t dk_cluster_id_x() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t dk_map_to_cta(uint32_t local_addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local_addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void dk_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void dk_st_cluster_f32(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void dk_st_cluster_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void dk_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void dk_wait_prerequisites() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void dk_report(int32_t* status, int code, int detail) {
    if (atomicCAS(status, 0, code) == 0) status[1] = detail;
}

// Ranges of the vocabulary that the head's gradient product is cut into (head.cu): the fewest k-steps of the busiest pair, where
// a further range costs its tiles' way through memory (512 KB at a pair's share of the bandwidth is about 22 steps of 64; a
// third of it shows beside the main loop), and no range is shorter than 4 steps.  A lane per number of ranges; the fewest win.
__device__ __forceinline__ int head_splits(const HeadEpilogue& h, int tiles, int steps, int lane) {
    const int s = lane + 1;
    int cost = 0x7fffffff;
    if (s == 1 || (tiles * s <= h.max_items && steps >= 4 * s))
        cost = (tiles * s + h.pairs - 1) / h.pairs * ((steps + s - 1) / s + 4) + (s > 1 ? s * tiles * 8 / h.pairs : 0);
    int best = cost, at = s;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const int c = __shfl_xor_sync(0xffffffffu, best, o), t = __shfl_xor_sync(0xffffffffu, at, o);
        if (c < best || (c == best && t < at)) { best = c; at = t; }
    }
    return at;
}

// ---- CTA pair (cta_group::2): loads that complete on the leader's barrier, MMA and commit for both CTAs ----
__device__ __forceinline__ void dg_tma_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster_addr, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster_addr), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void dg_tma_pair_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster_addr, int c0, int c1,
                                               int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster_addr), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void dg_commit_pair(uint32_t bar, uint16_t mask) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"(mask)
                 : "memory");
}
__device__ __forceinline__ void dg_mma_pair(uint32_t d_tmem, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
        : "memory");
}

}  // namespace sm100
}  // namespace marlaas
