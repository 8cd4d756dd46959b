// Stable order of a batch's tokens by a small key: by tenant (layer norm's gradients: every tenant's tokens one after another),
// or the tokens that a loss counts before those that it ignores.  A counting sort: each block of tokens counts its keys and
// ranks its tokens, one CTA turns the blocks' counts into positions, a third kernel places the tokens.  Integer work of 12
// bytes per token; a batch of one block takes all of it in one launch.
#include <string.h>

#include "sm100_cluster.cuh"

namespace marlaas {
using sm100::dk_report;

constexpr int ORDER_SMALL = 256, ORDER_LARGE = 1024;        // tokens per block: the large one while its counters fit 48 KB

// Key of token i: 0 .. cap - 1 its slot, cap for slot -1; or 0 for a token that counts, 1 for one that does not.
__device__ __forceinline__ int order_key(const OrderArgs& a, int64_t i) {
    if (a.targets) {
        const int t = a.targets[i];
        if (t >= a.V) dk_report(a.status, DEV_BAD_INDEX, (int)i);
        return t < 0 || t >= a.V || (a.weight && a.weight[i] == 0.f) ? 1 : 0;
    }
    int lo = 0, hi = a.S;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.off[mid + 1] > i) hi = mid; else lo = mid + 1;
    }
    const int t = lo < a.S ? a.slot[lo] : -1;
    if (t < -1 || t >= a.cap) dk_report(a.status, DEV_BAD_INDEX, (int)i);
    return t < 0 || t >= a.cap ? a.cap : t;
}

__device__ __forceinline__ void check_table(const OrderArgs& a) {
    for (int64_t s = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; s < a.S; s += (int64_t)gridDim.x * blockDim.x) {
        const int x = a.off[s], y = a.off[s + 1];
        if (y < x || x < 0 || y > a.T || (s == 0 && x != 0) || (s == a.S - 1 && y != a.T)) dk_report(a.status, DEV_BAD_TABLE, (int)s);
    }
}

// Exclusive sums of n counters in shared memory by one warp; the total goes to v[n].
__device__ __forceinline__ void warp_scan(int* v, int n) {
    const int lane = threadIdx.x & 31;
    int run = 0;
    for (int k0 = 0; k0 < n; k0 += 32) {
        const int x = k0 + lane < n ? v[k0 + lane] : 0;
        int inc = x;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += y;
        }
        if (k0 + lane < n) v[k0 + lane] = run + inc - x;
        run += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) v[n] = run;
}

__global__ void k_order_count(OrderArgs a) {
    extern __shared__ int s_cnt[];          // [warps][nkeys], then [nkeys + 1]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5, n = a.nkeys;
    int* s_tot = s_cnt + warps * n;
    sm100::dk_launch_dependents();          // (what follows waits before it reads the order)
    check_table(a);
    for (int k = tid; k < warps * n; k += blockDim.x) s_cnt[k] = 0;
    __syncthreads();
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + tid;
    const int key = i < a.T ? order_key(a, i) : -1;
    const unsigned same = __match_any_sync(0xffffffffu, key);
    const int before = __popc(same & ((1u << lane) - 1u));
    if (key >= 0 && before == 0) s_cnt[warp * n + key] = __popc(same);
    __syncthreads();
    for (int k = tid; k < n; k += blockDim.x) {
        int run = 0;
        for (int w = 0; w < warps; ++w) {
            const int v = s_cnt[w * n + k];
            s_cnt[w * n + k] = run;
            run += v;
        }
        s_tot[k] = run;
        if (gridDim.x > 1) a.hist[(size_t)blockIdx.x * n + k] = run;
    }
    __syncthreads();
    const int rank = key >= 0 ? s_cnt[warp * n + key] + before : 0;
    if (gridDim.x > 1) {
        if (key >= 0) a.keyrank[i] = key * ORDER_LARGE + rank;
        return;
    }
    if (warp == 0) warp_scan(s_tot, n);
    __syncthreads();
    if (key >= 0) a.perm[s_tot[key] + rank] = (int)i;
    for (int k = tid; k <= n; k += blockDim.x) a.key_off[k] = s_tot[k];
}

// One CTA: a warp per key turns the blocks' counts into exclusive sums, then every key gets its first position.
__global__ void __launch_bounds__(1024) k_order_scan(OrderArgs a, int nblk) {
    extern __shared__ int s_tot[];          // [nkeys + 1]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = a.nkeys;
    sm100::dk_wait_prerequisites();
    sm100::dk_launch_dependents();
    for (int k = warp; k < n; k += 32) {
        int run = 0;
        for (int b0 = 0; b0 < nblk; b0 += 32) {
            const int b = b0 + lane;
            const int x = b < nblk ? a.hist[(size_t)b * n + k] : 0;
            int inc = x;
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += y;
            }
            if (b < nblk) a.hist[(size_t)b * n + k] = run + inc - x;
            run += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) s_tot[k] = run;
    }
    __syncthreads();
    if (warp == 0) warp_scan(s_tot, n);
    __syncthreads();
    for (int k = threadIdx.x; k <= n; k += 1024) a.key_off[k] = s_tot[k];
}

__global__ void k_order_place(OrderArgs a) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    sm100::dk_wait_prerequisites();
    sm100::dk_launch_dependents();
    if (i >= a.T) return;
    const int kr = a.keyrank[i], key = kr / ORDER_LARGE, rank = kr % ORDER_LARGE;
    a.perm[a.key_off[key] + a.hist[(size_t)blockIdx.x * a.nkeys + key] + rank] = (int)i;
}

static int order_block(int nkeys) { return sizeof(int) * (size_t)(ORDER_LARGE / 32 + 1) * (nkeys + 1) <= 48 * 1024 ? ORDER_LARGE : ORDER_SMALL; }

size_t order_scratch_ints(int64_t T, int nkeys) { return (size_t)T + (size_t)cdiv(T, order_block(nkeys)) * nkeys; }

marlaas_status_t launch_order(const marlaas_pool* pool, OrderArgs a, int32_t* scratch, cudaStream_t st) {
    const int B = order_block(a.nkeys), nblk = (int)cdiv(a.T, B);
    a.keyrank = scratch;
    a.hist = scratch + a.T;
    a.status = pool->d_status;
    const size_t smem = sizeof(int) * ((size_t)(B / 32) * a.nkeys + a.nkeys + 1);
    if (smem > 48 * 1024) MARLAAS_CUDA_TRY(cudaFuncSetAttribute(k_order_count, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    k_order_count<<<nblk, B, smem, st>>>(a);
    MARLAAS_LAUNCH_CHECK("k_order_count");
    if (nblk == 1) return MARLAAS_OK;
    const marlaas_status_t rc = launch_link("k_order_scan", k_order_scan, dim3(1), 1024, sizeof(int) * ((size_t)a.nkeys + 1), true, st, a, nblk);
    return rc != MARLAAS_OK ? rc : launch_link("k_order_place", k_order_place, dim3((unsigned)nblk), (unsigned)B, 0, true, st, a);
}

}  // namespace marlaas
