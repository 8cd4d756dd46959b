// The policy update's calls on whole batches (Algorithm 1, training branch; Experimental setup: GRPO): group-relative
// advantages and token weights from rewards, token log-probabilities, the clipped policy loss.  The passes over the
// logits are in vocab_rows.cu.
#include <string.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "sm100_cluster.cuh"

namespace marlaas {

using sm100::dk_report;

// ---- group-relative advantages ----
// Three steps: active tokens per sequence and advantages per group; totals per tenant (integer sums, so their order does not
// matter); every token's advantage and weight.  They move 12 bytes per token: HBM for millions of tokens, launches for
// ordinary batches.  A small batch takes all three in one CTA and one launch (1024 tokens in 16 sequences: 4.1 us against
// 7.0 in two kernels; but 8192 tokens in 64: 9.1 against 6.3, and 16000 in 1000: 44 against 11).  A larger one counts in one
// kernel and expands in a second, each of whose CTAs forms the totals from the counts, and then every sequence's advantage
// and weight, for itself in shared memory; for more sequences than fit that way a kernel between them forms the totals (with
// 2000 sequences of 1000 tokens 15.1 us against 12.3).
constexpr int ADV_THREADS = 256, ADV_EXPAND_THREADS = 512, ADV_SMALL_THREADS = 1024;
constexpr int ADV_SMALL_T = 4096, ADV_SMALL_S = 128, ADV_SHARED_S = 2048, ADV_RUN = 512;

struct AdvArgs {
    int T, S, G, cap;
    const int32_t* off;
    const int32_t* slot;
    const int32_t* group_off;
    const int32_t* targets;
    const float* rewards;
    float eps;
    int token_mean, no_std;
    float* seq_adv;     // [S] always written (the caller's or the workspace's)
    float* adv;
    float* weight;
    int32_t* count;     // [S] active tokens
    int32_t* total;     // [cap + 1] active tokens, or sequences that have any, per bucket (of the kernel between)
    int32_t* status;
};

// First token and end of sequence s, inside [0, T] whatever the table holds.
__device__ __forceinline__ void seq_range(const AdvArgs& a, int s, int* lo, int* hi) {
    const int x = a.off[s], y = a.off[s + 1];
    *lo = min(max(x, 0), a.T);
    *hi = min(max(y, *lo), a.T);
}
__device__ __forceinline__ int bucket_of(const AdvArgs& a, int slot) { return slot < 0 || slot >= a.cap ? a.cap : slot; }
__device__ __forceinline__ void check_sequence(const AdvArgs& a, int s) {
    const int x = a.off[s], y = a.off[s + 1], t = a.slot[s];
    if (y < x || x < 0 || y > a.T || (s == 0 && x != 0) || (s == a.S - 1 && y != a.T)) dk_report(a.status, DEV_BAD_TABLE, s);
    if (t < -1 || t >= a.cap) dk_report(a.status, DEV_BAD_INDEX, s);
}
// Active tokens among [lo, hi) that lane `lane` of `lanes` looks at: whole 16-byte words in the middle, single tokens around.
__device__ __forceinline__ int count_active(const int32_t* targets, int lo, int hi, int lane, int lanes) {
    const int head = (int)(((16 - ((uintptr_t)(targets + lo) & 15)) & 15) >> 2), mid = min(lo + head, hi), words = (hi - mid) >> 2;
    int n = 0;
    if (lane < mid - lo) n += targets[lo + lane] >= 0;
    const int4* w = reinterpret_cast<const int4*>(targets + mid);
#pragma unroll 4
    for (int i = lane; i < words; i += lanes) {
        const int4 t = w[i];
        n += (t.x >= 0) + (t.y >= 0) + (t.z >= 0) + (t.w >= 0);
    }
    const int tail = mid + 4 * words;       // (compared with what is left: tail + lane may pass 2^31)
    if (lane < hi - tail) n += targets[tail + lane] >= 0;
    return n;
}
__device__ __forceinline__ int warp_total(int n) { return __reduce_add_sync(0xffffffffu, n); }

// One warp: the advantages of group g's sequences.
__device__ __forceinline__ void group_advantages(const AdvArgs& a, int g, int lane, float* seq_adv) {
    const int x = a.group_off[g], y = a.group_off[g + 1];
    if (lane == 0 && (y < x || x < 0 || y > a.S || (g == 0 && x != 0) || (g == a.G - 1 && y != a.S)))
        dk_report(a.status, DEV_BAD_TABLE, -10 - g);
    const int lo = min(max(x, 0), a.S), hi = min(max(y, lo), a.S);
    if (hi <= lo) return;
    // differences to the group's first reward: rewards that are all alike give exact zeros
    const float r0 = a.rewards[lo], n = (float)(hi - lo);
    float sum = 0.f;
    for (int i = lo + lane; i < hi; i += 32) sum += a.rewards[i] - r0;
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float mean = sum / n;
    float sq = 0.f;
    if (!a.no_std) {
        for (int i = lo + lane; i < hi; i += 32) {
            const float d = (a.rewards[i] - r0) - mean;
            sq += d * d;
        }
        for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
    }
    const float sd = sqrtf(sq / n);
    for (int i = lo + lane; i < hi; i += 32) {
        const float d = (a.rewards[i] - r0) - mean, v = a.no_std ? d : (d == 0.f ? 0.f : d / (sd + a.eps));      // (eps may be 0)
        seq_adv[i] = v;
        if (seq_adv != a.seq_adv) a.seq_adv[i] = v;
    }
}
__device__ __forceinline__ float token_weight(const AdvArgs& a, int count, int total) {
    return count == 0 ? 0.f : 1.f / (a.token_mean ? (float)total : (float)total * (float)count);
}

__global__ void __launch_bounds__(ADV_SMALL_THREADS) k_adv_small(const AdvArgs a) {
    extern __shared__ int32_t s_total[];                    // [cap + 1]
    __shared__ float s_adv[ADV_SMALL_S], s_weight[ADV_SMALL_S];
    __shared__ int32_t s_count[ADV_SMALL_S], s_off[ADV_SMALL_S];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int b = tid; b <= a.cap; b += ADV_SMALL_THREADS) s_total[b] = 0;
    if (tid < a.S) {
        s_adv[tid] = 0.f;       // (a table that leaves a sequence out)
        s_off[tid] = a.off[tid];
    }
    __syncthreads();
    for (int s = warp; s < a.S; s += ADV_SMALL_THREADS / 32) {
        int lo, hi;
        seq_range(a, s, &lo, &hi);
        const int n = warp_total(count_active(a.targets, lo, hi, lane, 32));
        if (lane == 0) {
            check_sequence(a, s);
            s_count[s] = n;
            if (n) atomicAdd(s_total + bucket_of(a, a.slot[s]), a.token_mean ? n : 1);
        }
    }
    for (int g = warp; g < a.G; g += ADV_SMALL_THREADS / 32) group_advantages(a, g, lane, s_adv);
    __syncthreads();
    if (tid < a.S) s_weight[tid] = token_weight(a, s_count[tid], s_total[bucket_of(a, a.slot[tid])]);
    __syncthreads();
    for (int i = tid; i < a.T; i += ADV_SMALL_THREADS) {
        int lo = 0, hi = a.S;           // sequences that begin at or before the token: the last of them holds it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_off[mid] <= i) lo = mid + 1; else hi = mid;
        }
        const bool on = lo > 0 && a.targets[i] >= 0;
        if (a.adv) a.adv[i] = on ? s_adv[lo - 1] : 0.f;
        if (a.weight) a.weight[i] = on ? s_weight[lo - 1] : 0.f;
    }
}

// WPS warps per sequence count its active tokens; then one warp per group.
template <int WPS>
__global__ void __launch_bounds__(ADV_THREADS) k_adv_count(const AdvArgs a) {
    __shared__ int s_n[ADV_THREADS / 32];
    constexpr int TEAMS = ADV_THREADS / 32 / WPS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team = warp / WPS;
    sm100::dk_launch_dependents();
    for (int s0 = blockIdx.x * TEAMS; s0 < a.S; s0 += gridDim.x * TEAMS) {
        const int s = s0 + team;
        int n = 0;
        if (s < a.S) {
            int lo, hi;
            seq_range(a, s, &lo, &hi);
            n = warp_total(count_active(a.targets, lo, hi, threadIdx.x % (32 * WPS), 32 * WPS));
        }
        if (WPS > 1) {
            if (lane == 0) s_n[warp] = n;
            __syncthreads();
            if (warp % WPS == 0)
                for (int w = 1; w < WPS; ++w) n += s_n[warp + w];
            __syncthreads();
        }
        if (s < a.S && warp % WPS == 0 && lane == 0) {
            check_sequence(a, s);
            a.count[s] = n;
        }
    }
    for (int g = (int)gridDim.x - 1 - (int)blockIdx.x + (int)gridDim.x * warp; g < a.G; g += (int)gridDim.x * (ADV_THREADS / 32))
        group_advantages(a, g, lane, a.seq_adv);
}

__global__ void __launch_bounds__(1024) k_adv_totals(const AdvArgs a) {
    for (int b = threadIdx.x; b <= a.cap; b += 1024) a.total[b] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < a.S; s += 1024) {
        const int n = a.count[s];
        if (n) atomicAdd(a.total + bucket_of(a, a.slot[s]), a.token_mean ? n : 1);
    }
}

// A warp takes a run of ADV_RUN tokens, four per lane at a time; the sequence of the run's first token by bisection, the
// others' from there on.
template <bool SHARED>
__global__ void __launch_bounds__(ADV_EXPAND_THREADS) k_adv_expand(const AdvArgs a) {
    extern __shared__ float2 s_seq[];       // SHARED: [S] advantage and weight, then [cap + 1] totals, [S] offsets
    const int tid = threadIdx.x;
    int32_t* s_total = reinterpret_cast<int32_t*>(s_seq + a.S);
    int32_t* s_off = s_total + a.cap + 1;
    if (SHARED) {
        for (int b = tid; b <= a.cap; b += ADV_EXPAND_THREADS) s_total[b] = 0;
        for (int s = tid; s < a.S; s += ADV_EXPAND_THREADS) s_off[s] = a.off[s];
        __syncthreads();
        sm100::dk_wait_prerequisites();
        for (int s0 = 0; s0 < a.S; s0 += ADV_EXPAND_THREADS) {
            const int s = s0 + tid, n = s < a.S ? a.count[s] : 0, b = s < a.S ? bucket_of(a, a.slot[s]) : a.cap;
            const int add = n ? (a.token_mean ? n : 1) : 0;
            if (__all_sync(0xffffffffu, b == __shfl_sync(0xffffffffu, b, 0))) {     // a tenant's sequences side by side
                const int sum = warp_total(add);
                if ((tid & 31) == 0 && sum) atomicAdd(s_total + b, sum);
            } else if (add) {
                atomicAdd(s_total + b, add);
            }
        }
        __syncthreads();
        for (int s = tid; s < a.S; s += ADV_EXPAND_THREADS)
            s_seq[s] = make_float2(a.seq_adv[s], token_weight(a, a.count[s], s_total[bucket_of(a, a.slot[s])]));
        __syncthreads();
    }
    const int32_t* off = SHARED ? s_off : a.off;
    const bool wide = ((((uintptr_t)a.targets | (uintptr_t)a.adv | (uintptr_t)a.weight)) & 15) == 0;
    const int lane = tid & 31;
    const int64_t warps = (int64_t)gridDim.x * (ADV_EXPAND_THREADS / 32);
    for (int64_t w = ((int64_t)blockIdx.x * ADV_EXPAND_THREADS + tid) >> 5; w * ADV_RUN < a.T; w += warps) {
        const int begin = (int)(w * ADV_RUN), end = min(a.T - begin, ADV_RUN) + begin;
        int4 t[ADV_RUN / 128];
#pragma unroll
        for (int j = 0; j < ADV_RUN / 128; ++j) {
            const int i = 128 * j + 4 * lane, n = end - begin - i;         // tokens from this thread's first on
            t[j] = make_int4(-1, -1, -1, -1);
            if (wide && n >= 4) {
                t[j] = *reinterpret_cast<const int4*>(a.targets + begin + i);
            } else {
                if (n > 0) t[j].x = a.targets[begin + i];
                if (n > 1) t[j].y = a.targets[begin + i + 1];
                if (n > 2) t[j].z = a.targets[begin + i + 2];
                if (n > 3) t[j].w = a.targets[begin + i + 3];
            }
        }
        int lo = 0, hi = a.S;               // sequences that begin at or before the run: the last of them holds its first token
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (off[mid] <= begin) lo = mid + 1; else hi = mid;
        }
        int s = lo - 1;
#pragma unroll
        for (int j = 0; j < ADV_RUN / 128; ++j) {
            const int step = 128 * j, i = step + 4 * lane, n = end - begin - i;
            if (begin + step >= end) break;
            while (s + 1 < a.S && off[s + 1] <= begin + step) ++s;
            const bool on[4] = {t[j].x >= 0, t[j].y >= 0, t[j].z >= 0, t[j].w >= 0};
            float va[4], wa[4];
            auto values = [&](int q) {
                if (q < 0) return make_float2(0.f, 0.f);
                if (SHARED) return s_seq[q];
                return make_float2(a.seq_adv[q], token_weight(a, a.count[q], a.total[bucket_of(a, a.slot[q])]));
            };
            if (s + 1 >= a.S || off[s + 1] - begin >= step + 128) {        // all 128 tokens are of one sequence
                const float2 vw = values(s);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    va[k] = on[k] ? vw.x : 0.f;
                    wa[k] = on[k] ? vw.y : 0.f;
                }
            } else {
                int q = s;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    while (k < n && q + 1 < a.S && off[q + 1] <= begin + i + k) ++q;       // (sequences may be empty)
                    const float2 vw = on[k] ? values(q) : make_float2(0.f, 0.f);
                    va[k] = vw.x;
                    wa[k] = vw.y;
                }
            }
            if (wide && n >= 4) {
                if (a.adv) *reinterpret_cast<float4*>(a.adv + begin + i) = make_float4(va[0], va[1], va[2], va[3]);
                if (a.weight) *reinterpret_cast<float4*>(a.weight + begin + i) = make_float4(wa[0], wa[1], wa[2], wa[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k < n && a.adv) a.adv[begin + i + k] = va[k];
                    if (k < n && a.weight) a.weight[begin + i + k] = wa[k];
                }
            }
        }
    }
}

static marlaas_status_t launch_advantages(const marlaas_pool* pool, const AdvArgs& a, cudaStream_t st) {
    if (a.T <= ADV_SMALL_T && a.S <= ADV_SMALL_S) {
        k_adv_small<<<1, ADV_SMALL_THREADS, sizeof(int32_t) * ((size_t)a.cap + 1), st>>>(a);
        MARLAAS_LAUNCH_CHECK("k_adv_small");
        return MARLAAS_OK;
    }
    const int64_t most = (int64_t)pool->sm_count * (2048 / ADV_THREADS);
    // long sequences: four warps each (64 of 4096 tokens: 7.0 us against 9.1 with one; 1000 of 256 or fewer: the same)
    const bool long_ones = a.T / a.S > 256;
    const int64_t teams = long_ones ? ADV_THREADS / 128 : ADV_THREADS / 32;
    const int grid = (int)std::min<int64_t>(std::max<int64_t>(cdiv(a.S, teams), cdiv(a.G, ADV_THREADS / 32)), most);
    if (long_ones) k_adv_count<4><<<grid, ADV_THREADS, 0, st>>>(a);
    else k_adv_count<1><<<grid, ADV_THREADS, 0, st>>>(a);
    MARLAAS_LAUNCH_CHECK("k_adv_count");
    if (!a.adv && !a.weight) return MARLAAS_OK;
    const int egrid = (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(a.T, (int64_t)ADV_EXPAND_THREADS / 32 * ADV_RUN), (int64_t)pool->sm_count * 4));
    if (a.S <= ADV_SHARED_S) {
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof(cfg));
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((unsigned)egrid);
        cfg.blockDim = dim3(ADV_EXPAND_THREADS);
        cfg.dynamicSmemBytes = sizeof(float2) * (size_t)a.S + sizeof(int32_t) * ((size_t)a.cap + 1 + a.S);
        cfg.stream = st;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        MARLAAS_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_adv_expand<true>, a));
    } else {
        k_adv_totals<<<1, 1024, 0, st>>>(a);
        MARLAAS_LAUNCH_CHECK("k_adv_totals");
        k_adv_expand<false><<<egrid, ADV_EXPAND_THREADS, 0, st>>>(a);
    }
    MARLAAS_LAUNCH_CHECK("k_adv_expand");
    return MARLAAS_OK;
}

// One CTA per bucket sums its tokens' terms, every thread its own tokens in ascending order, then a fixed tree.  A token's
// segment is found by bisection, in a copy of the offsets in shared memory where they fit.  Every bucket with a segment looks at
// all tokens: beside wide rows that does not show, for hundreds of tenants over short rows it does (the loss over 4096 x 1000
// takes 20 us for up to 128 tenants, 33 for 512; over 65536 x 1000 175 to 190, and 341).
constexpr int STATS_THREADS = 1024, STATS_OFFSETS = 4096;
__global__ void __launch_bounds__(STATS_THREADS) k_policy_stats(int T, int S, int cap, const int32_t* __restrict__ seg_offsets,
                                                                const int32_t* __restrict__ seg_slot, const PolicyTerms* __restrict__ terms,
                                                                float* __restrict__ stats, int accumulate, int32_t* status) {
    __shared__ float s_sum[32][MARLAAS_POLICY_STATS];
    __shared__ int32_t s_off[STATS_OFFSETS];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // launched while the rows kernel runs: the tables are there, the terms are not
    const bool cached = S < STATS_OFFSETS;
    bool mine = b == cap;           // (tokens that an ill-formed table leaves out count there)
    for (int s = tid; s < S; s += STATS_THREADS) {
        const int x = seg_offsets[s], y = seg_offsets[s + 1], t = seg_slot[s];
        if (cached) s_off[s] = x;
        mine |= t == b;
        if (b == 0) {
            if (y < x || x < 0 || y > T || (s == 0 && x != 0) || (s == S - 1 && y != T)) dk_report(status, DEV_BAD_TABLE, s);
            if (t < -1 || t >= cap) dk_report(status, DEV_BAD_INDEX, s);
        }
    }
    const bool any = __syncthreads_or(mine) != 0;
    sm100::dk_wait_prerequisites();
    if (!any) {
        if (tid < MARLAAS_POLICY_STATS && !accumulate) stats[(size_t)b * MARLAAS_POLICY_STATS + tid] = 0.f;
        return;
    }
    const int32_t* off = cached ? s_off : seg_offsets;
    float v[MARLAAS_POLICY_STATS] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t i = tid; i < T; i += STATS_THREADS) {
        int lo = 0, hi = S;         // segments that begin at or before the token: the last of them holds it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (off[mid] <= i) lo = mid + 1; else hi = mid;
        }
        const int t = lo > 0 ? seg_slot[lo - 1] : -1;
        if ((t < 0 || t >= cap ? cap : t) != b) continue;
        const float4 x = reinterpret_cast<const float4*>(terms + i)[0], y = reinterpret_cast<const float4*>(terms + i)[1];
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
    }
#pragma unroll
    for (int k = 0; k < MARLAAS_POLICY_STATS; ++k)
        for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (lane == 0)
#pragma unroll
        for (int k = 0; k < MARLAAS_POLICY_STATS; ++k) s_sum[warp][k] = v[k];
    __syncthreads();
    if (tid < MARLAAS_POLICY_STATS) {
        float x = 0.f;
        for (int w = 0; w < 32; ++w) x += s_sum[w][tid];
        float* out = stats + (size_t)b * MARLAAS_POLICY_STATS + tid;
        *out = accumulate ? *out + x : x;
    }
}

// Segment and group tables on the device.
struct PolicyTables {
    const int32_t* off;
    const int32_t* slot;
    const int32_t* group_off;
};

// Workspace of the two calls that need one.
struct PolicyWorkspace {
    PolicyTerms* terms;     // [T]
    int32_t* off;           // [S + 1] host tables, staged by one copy
    int32_t* slot;          // [S]
    int32_t* group_off;     // [G + 1]
    int32_t* count;         // [S]
    int32_t* total;         // [cap + 1]
    float* seq_adv;         // [S]
    size_t total_bytes;
};
static PolicyWorkspace carve_policy(const marlaas_pool* pool, int64_t T, int32_t S, int32_t G, void* base) {
    PolicyWorkspace w;
    char* p = (char*)base;
    size_t o = 0;
    auto take = [&](size_t bytes) { char* q = p ? p + o : nullptr; o += align_up(bytes, 256); return q; };
    w.terms = (PolicyTerms*)take(sizeof(PolicyTerms) * (size_t)T);
    w.off = (int32_t*)take(sizeof(int32_t) * ((size_t)S + 1));
    w.slot = (int32_t*)take(sizeof(int32_t) * (size_t)S);
    w.group_off = (int32_t*)take(sizeof(int32_t) * ((size_t)G + 1));
    w.count = (int32_t*)take(sizeof(int32_t) * (size_t)S);
    w.total = (int32_t*)take(sizeof(int32_t) * ((size_t)pool->cap + 1));
    w.seq_adv = (float*)take(sizeof(float) * (size_t)S);
    w.total_bytes = o;
    return w;
}

// Host tables into the workspace, whose arrays for them lie one after another, by one copy.  Its source is a vector of the
// call's own: pageable, so the runtime has staged it when the copy returns, and the caller's tables may be page-locked memory that
// is written again after the call.
static marlaas_status_t stage_tables(const marlaas_segments_t* seg, int32_t num_groups, const int32_t* group_offsets,
                                     const PolicyWorkspace& ws, PolicyTables* t, cudaStream_t st) {
    const size_t S = (size_t)seg->num_segments;
    const int32_t* end = group_offsets ? ws.group_off + num_groups + 1 : ws.slot + S;
    std::vector<int32_t> copy((size_t)(end - ws.off));
    std::copy(seg->seg_offsets, seg->seg_offsets + S + 1, copy.begin());
    std::copy(seg->seg_slot, seg->seg_slot + S, copy.begin() + (ws.slot - ws.off));
    if (group_offsets) std::copy(group_offsets, group_offsets + num_groups + 1, copy.begin() + (ws.group_off - ws.off));
    MARLAAS_CUDA_TRY(cudaMemcpyAsync(ws.off, copy.data(), sizeof(int32_t) * copy.size(), cudaMemcpyHostToDevice, st));
    *t = PolicyTables{ws.off, ws.slot, ws.group_off};
    return MARLAAS_OK;
}

static bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

static marlaas_status_t check_rows(const char* fn, const char* name, const void* p, int64_t ld, int64_t V, int32_t dtype) {
    const int64_t per16 = dtype == MARLAAS_DTYPE_F32 ? 4 : 8;
    if (!p || misaligned(p, 16)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: %s is NULL or not 16-byte aligned", fn, name);
    if (ld < V || ld % per16 != 0 || ld >= (1ll << 31))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: leading dimension of %s (%lld) must be >= %lld and a multiple of %lld", fn, name,
                    (long long)ld, (long long)V, (long long)per16);
    return MARLAAS_OK;
}

// The arguments that token_logprobs and policy_loss have in common.
static marlaas_status_t check_logits(const char* fn, const marlaas_pool* pool, int64_t T, int64_t V, const void* logits,
                                     int64_t ld, int32_t dtype, const int32_t* targets, float inv_temperature) {
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (T < 0 || T >= (1ll << 31)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: T out of range", fn);
    if (V < 1 || V > MARLAAS_MAX_VOCABULARY)
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: V = %lld outside [1, %d]", fn, (long long)V, (int)MARLAAS_MAX_VOCABULARY);
    if (dtype != MARLAAS_DTYPE_BF16 && dtype != MARLAAS_DTYPE_F32) return fail(MARLAAS_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)dtype);
    if (!(inv_temperature > 0.f) || !std::isfinite(2.f * inv_temperature))       // (it is scaled by 1 / ln 2)
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: inv_temperature must be positive, finite and below 1.7e38", fn);
    if (T == 0) return MARLAAS_OK;
    if (!targets || misaligned(targets, 4)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: targets is NULL or misaligned", fn);
    return check_rows(fn, "logits", logits, ld, V, dtype);
}

}  // namespace marlaas

using namespace marlaas;

extern "C" {

size_t marlaas_policy_workspace_bytes(const marlaas_pool_t* pool, int64_t T, int32_t num_segments, int32_t num_groups) {
    if (!pool || T < 0 || T >= (1ll << 31) || num_segments < 0 || num_segments > MAX_SEGMENTS || num_groups < 0 || num_groups > MAX_SEGMENTS)
        return 0;
    return carve_policy(pool, T, num_segments, num_groups, nullptr).total_bytes;
}

marlaas_status_t marlaas_group_advantages(marlaas_pool_t* pool, int64_t T, const marlaas_segments_t* seg, const float* rewards,
                                          int32_t num_groups, const int32_t* group_offsets, const int32_t* targets, float eps,
                                          float* seq_adv, float* adv, float* weight, void* workspace, size_t workspace_bytes,
                                          uint32_t flags, void* cuda_stream) try {
    const char* fn = "group_advantages";
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (T < 0 || T >= (1ll << 31)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: T out of range", fn);
    if (flags & ~(uint32_t)(MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC | MARLAAS_FLAG_TOKEN_MEAN | MARLAAS_FLAG_NO_STD))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: a flag does not apply to this call", fn);
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: eps must be finite and not negative", fn);
    if (num_groups < 0 || num_groups > MAX_SEGMENTS)
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: group count outside [0, %d]", fn, (int)MAX_SEGMENTS);
    marlaas_status_t rc = check_segments(fn, pool, T, seg, flags, nullptr);
    if (rc != MARLAAS_OK) return rc;
    const int32_t S = seg->num_segments;
    if (S > 0 && (num_groups == 0 || !group_offsets))
        return fail(MARLAAS_ERR_BAD_SEGMENT_TABLE, "%s: empty group table for %d sequences", fn, S);
    if (S > 0 && (!seg->seg_offsets || !seg->seg_slot)) return fail(MARLAAS_ERR_BAD_SEGMENT_TABLE, "%s: segment arrays are NULL", fn);
    const bool host = (flags & MARLAAS_FLAG_HOST_TABLE) != 0;
    if (host && S > 0) {
        if (group_offsets[0] != 0 || group_offsets[num_groups] != S)
            return fail(MARLAAS_ERR_BAD_SEGMENT_TABLE, "%s: group_offsets must run from 0 to %d", fn, S);
        for (int32_t g = 0; g < num_groups; ++g)
            if (group_offsets[g + 1] < group_offsets[g])
                return fail(MARLAAS_ERR_BAD_SEGMENT_TABLE, "%s: group_offsets decreases at group %d", fn, g);
    }
    if (S > 0 && (!rewards || misaligned(rewards, 4))) return fail(MARLAAS_ERR_INVALID_ARG, "%s: rewards is NULL or misaligned", fn);
    if (T > 0 && (!targets || misaligned(targets, 4))) return fail(MARLAAS_ERR_INVALID_ARG, "%s: targets is NULL or misaligned", fn);
    if (misaligned(seq_adv, 4) || misaligned(adv, 4) || misaligned(weight, 4))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: an output is misaligned", fn);
    if (S == 0) return MARLAAS_OK;
    if (!workspace || misaligned(workspace, 256)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: workspace NULL or misaligned", fn);
    const PolicyWorkspace ws = carve_policy(pool, T, S, num_groups, workspace);
    if (workspace_bytes < ws.total_bytes)
        return fail(MARLAAS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < required %zu", fn, workspace_bytes, ws.total_bytes);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    AdvArgs a;
    a.T = (int)T; a.S = S; a.G = num_groups; a.cap = pool->cap;
    PolicyTables t = {seg->seg_offsets, seg->seg_slot, group_offsets};
    if (host && (rc = stage_tables(seg, num_groups, group_offsets, ws, &t, st)) != MARLAAS_OK) return rc;
    a.off = t.off; a.slot = t.slot; a.group_off = t.group_off;
    a.targets = targets; a.rewards = rewards; a.eps = eps;
    a.token_mean = (flags & MARLAAS_FLAG_TOKEN_MEAN) != 0; a.no_std = (flags & MARLAAS_FLAG_NO_STD) != 0;
    a.seq_adv = seq_adv ? seq_adv : ws.seq_adv;
    a.adv = adv; a.weight = weight; a.count = ws.count; a.total = ws.total; a.status = pool->d_status;
    if ((rc = launch_advantages(pool, a, st)) != MARLAAS_OK) return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "group_advantages: %s", e.what());
}

marlaas_status_t marlaas_token_logprobs(marlaas_pool_t* pool, int64_t T, int64_t V, const void* logits, int64_t ld, int32_t dtype,
                                        const int32_t* targets, float inv_temperature, float* logp, float* entropy,
                                        uint32_t flags, void* cuda_stream) {
    const char* fn = "token_logprobs";
    marlaas_status_t rc = check_logits(fn, pool, T, V, logits, ld, dtype, targets, inv_temperature);
    if (rc != MARLAAS_OK) return rc;
    if (flags & ~(uint32_t)MARLAAS_FLAG_VALIDATE_SYNC) return fail(MARLAAS_ERR_INVALID_ARG, "%s: a flag does not apply to this call", fn);
    if (T == 0) return MARLAAS_OK;
    if (!logp || misaligned(logp, 4) || misaligned(entropy, 4))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: logp is NULL or an output is misaligned", fn);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    VocabRows r;
    memset(&r, 0, sizeof(r));
    r.T = T; r.V = V; r.logits = logits; r.ld = ld; r.f32 = dtype == MARLAAS_DTYPE_F32;
    r.targets = targets; r.inv_temperature = inv_temperature; r.logp = logp; r.entropy = entropy; r.status = pool->d_status;
    if ((rc = launch_vocab_rows(pool, r, st)) != MARLAAS_OK) return rc;
    return finish(pool, flags, st);
}

marlaas_status_t marlaas_policy_loss(marlaas_pool_t* pool, int64_t T, int64_t V, const void* logits, int64_t ld, int32_t dtype,
                                     const int32_t* targets, const marlaas_segments_t* seg, const float* old_logp,
                                     const float* ref_logp, const float* adv, const float* weight,
                                     const marlaas_policy_loss_t* hp, void* dlogits, int64_t lddl, float* logp, float* stats,
                                     void* workspace, size_t workspace_bytes, uint32_t flags, void* cuda_stream) try {
    const char* fn = "policy_loss";
    if (!hp) return fail(MARLAAS_ERR_INVALID_ARG, "%s: the loss's parameters are NULL", fn);
    marlaas_status_t rc = check_logits(fn, pool, T, V, logits, ld, dtype, targets, hp->inv_temperature);
    if (rc != MARLAAS_OK) return rc;
    if (flags & ~(uint32_t)(MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC | MARLAAS_FLAG_ACCUMULATE))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: a flag does not apply to this call", fn);
    if (!(hp->clip_low >= 0.f) || !(hp->clip_high >= 0.f))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: clip_low and clip_high must not be negative", fn);
    if (!std::isfinite(hp->kl_coef) || !std::isfinite(hp->entropy_coef) || !std::isfinite(hp->grad_scale))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: a coefficient is not finite", fn);
    if (!stats || misaligned(stats, 4) || misaligned(logp, 4)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: stats is NULL or an output is misaligned", fn);
    if (logp && (logp == old_logp || logp == ref_logp || logp == adv || logp == weight))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: logp must not be one of the inputs", fn);
    if ((rc = check_segments(fn, pool, T, seg, flags, nullptr)) != MARLAAS_OK) return rc;
    const bool accumulate = (flags & MARLAAS_FLAG_ACCUMULATE) != 0;
    PolicyWorkspace ws;
    memset(&ws, 0, sizeof(ws));
    if (T > 0) {
        if (!old_logp || !adv || !weight || misaligned(old_logp, 4) || misaligned(adv, 4) || misaligned(weight, 4) || misaligned(ref_logp, 4))
            return fail(MARLAAS_ERR_INVALID_ARG, "%s: old_logp, adv or weight is NULL, or an input is misaligned", fn);
        if (!ref_logp && hp->kl_coef != 0.f) return fail(MARLAAS_ERR_INVALID_ARG, "%s: ref_logp is NULL although kl_coef is not 0", fn);
        if (dlogits) {
            if ((rc = check_rows(fn, "dlogits", dlogits, lddl, V, dtype)) != MARLAAS_OK) return rc;
            const size_t e = dtype == MARLAAS_DTYPE_F32 ? 4 : 2;
            const uintptr_t z0 = (uintptr_t)logits, z1 = z0 + ((size_t)(T - 1) * ld + V) * e;
            const uintptr_t d0 = (uintptr_t)dlogits, d1 = d0 + ((size_t)(T - 1) * lddl + V) * e;
            if (d0 < z1 && z0 < d1 && !(d0 == z0 && lddl == ld))
                return fail(MARLAAS_ERR_INVALID_ARG, "%s: dlogits overlaps logits without being the same matrix", fn);
        }
        if (!workspace || misaligned(workspace, 256)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: workspace NULL or misaligned", fn);
        ws = carve_policy(pool, T, seg->num_segments, 0, workspace);
        if (workspace_bytes < ws.total_bytes)
            return fail(MARLAAS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < required %zu", fn, workspace_bytes, ws.total_bytes);
    }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    PolicyTables t = {seg->seg_offsets, seg->seg_slot, nullptr};
    if (T > 0) {
        if ((flags & MARLAAS_FLAG_HOST_TABLE) && (rc = stage_tables(seg, 0, nullptr, ws, &t, st)) != MARLAAS_OK) return rc;
        VocabRows r;
        memset(&r, 0, sizeof(r));
        r.T = T; r.V = V; r.logits = logits; r.ld = ld; r.f32 = dtype == MARLAAS_DTYPE_F32;
        r.targets = targets; r.inv_temperature = hp->inv_temperature; r.logp = logp; r.terms = ws.terms;
        r.old_logp = old_logp; r.ref_logp = ref_logp; r.adv = adv; r.weight = weight;
        r.clip_low = hp->clip_low; r.clip_high = hp->clip_high; r.kl_coef = hp->kl_coef; r.entropy_coef = hp->entropy_coef;
        r.grad_scale = hp->grad_scale; r.dlogits = dlogits; r.lddl = lddl; r.status = pool->d_status;
        if ((rc = launch_vocab_rows(pool, r, st)) != MARLAAS_OK) return rc;
    }
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)(pool->cap + 1));
    cfg.blockDim = dim3(STATS_THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    MARLAAS_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_policy_stats, (int)T, T > 0 ? (int)seg->num_segments : 0, (int)pool->cap, t.off, t.slot,
                                        (const PolicyTerms*)ws.terms, stats, (int)accumulate, pool->d_status));
    MARLAAS_LAUNCH_CHECK("k_policy_stats");
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "policy_loss: %s", e.what());
}

}  // extern "C"
