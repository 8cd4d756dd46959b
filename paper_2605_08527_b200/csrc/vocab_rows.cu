// Rows of logits: log-probability of the target, entropy, the clipped policy loss's terms and the gradient by the logits
// (Algorithm 1: "PolicyUpdate"; Experimental setup: GRPO).  With z the row, k = inv_temperature:
//     m = max z    s = sum exp((z - m) k)    logp = (z_a - m) k - log s    H = log s - sum p (z - m) k
//     dz_j = g ( p_j (c_H (log p_j + H) - c) + [j = a] c ),   g = grad_scale w k,   c = d(pg + kl_coef kl) / d logp
#include <math.h>
#include <string.h>

#include <atomic>

#include "sm100_cluster.cuh"

namespace marlaas {
using namespace sm100;

constexpr int MAX_DEVICES = 16;
constexpr float VR_LOG2E = 1.4426950408889634f, VR_LN2 = 0.6931471805599453f;

// max that keeps a NaN (fmaxf drops it): a bad logit has to show in the row's outputs
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Powers and logarithms of 2 by the special-function unit: a relative error of 2^-22 for the powers, an absolute one of
// 2^-22 for the logarithm of a row's sum, 2e-7 of a log-probability of order 10.
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float lg2(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The reference point of a running maximum: 0 while there is no finite logit, so that -inf - m stays -inf.
__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }
// (z - m) k in units of log 2, not below -200: 2^-200 is 0 in fp32, and a product with it stays 0 where (z - m) k itself is
// -inf.  The difference comes first: z k alone may leave fp32's range where a mask is the type's lowest value.
__device__ __forceinline__ float exponent(float z, float m, float k2) { return max_nan((z - m) * k2, -200.f); }

template <bool F32>
struct Vec;
template <>
struct Vec<false> {     // 8 bf16 in 16 bytes
    static constexpr int N = 8;
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[4]) {
        uint4 q;
        uint32_t* w = &q.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 p = __floats2bfloat162_rn(f[i].x, f[i].y);
            w[i] = *reinterpret_cast<uint32_t*>(&p);
        }
        return q;
    }
    static __device__ __forceinline__ float load(const void* p, int64_t i) { return __bfloat162float(((const bf16*)p)[i]); }
    static __device__ __forceinline__ void store(void* p, int64_t i, float v) { ((bf16*)p)[i] = __float2bfloat16_rn(v); }
};
template <>
struct Vec<true> {
    static constexpr int N = 4;
    static __device__ __forceinline__ uint4 pack(const float2 (&f)[2]) {
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    }
    static __device__ __forceinline__ float load(const void* p, int64_t i) { return ((const float*)p)[i]; }
    static __device__ __forceinline__ void store(void* p, int64_t i, float v) { ((float*)p)[i] = v; }
};

// What a row's gradient needs: dz_j = 2^(t_j - log2 s) (alpha t_j + beta), and + gamma at the target.
struct RowGrad {
    float alpha, beta, gamma;
};

// A token's inputs of the loss, loaded while its row is on the way.
struct TokenIn {
    float old, ref, A, w;
};

// The token's loss terms from its log-probability and entropy; the coefficients of its gradient.
__device__ __forceinline__ RowGrad token_terms(const VocabRows& a, const TokenIn& in, float logp, float H, float log2s, PolicyTerms* out) {
    const float w = in.w, A = in.A;
    const float ratio = ex2((logp - in.old) * VR_LOG2E);
    // 0 A is 0 whatever the ratio
    const float plain = A == 0.f ? 0.f : ratio * A;
    const float clipped = A == 0.f ? 0.f : fminf(fmaxf(ratio, 1.f - a.clip_low), 1.f + a.clip_high) * A;
    const bool is_clipped = plain > clipped;      // (a NaN counts as not clipped and shows in the loss)
    const float pg = -(is_clipped ? clipped : plain);
    float c = is_clipped ? 0.f : -plain, kl = 0.f, reg = pg;
    if (a.ref_logp) {       // the column is filled also where the loss has no such term
        const float d = in.ref - logp, e1 = expm1f(d);     // exp(d) - d - 1 without its cancellation for small d
        kl = d > 80.f ? e1 : e1 - d;        // (both may be infinite)
        if (a.kl_coef != 0.f) {
            c = fmaf(-a.kl_coef, e1, c);
            reg = fmaf(a.kl_coef, kl, pg);
        }
    }
    PolicyTerms t;
    t.loss = w * fmaf(-a.entropy_coef, H, reg);
    t.pg = w * pg; t.kl = w * kl; t.entropy = w * H; t.ratio = w * ratio;
    t.clipped = is_clipped ? w : 0.f;
    t.weight = w;
    t.count = 1.f;
    *out = t;
    // log p_j = (t_j - log2 s) ln 2
    const float g = a.grad_scale * w * a.inv_temperature;
    RowGrad r;
    r.alpha = g * a.entropy_coef * VR_LN2;
    r.beta = g * (a.entropy_coef * (H - log2s * VR_LN2) - c);
    r.gamma = g * c;
    return r;
}

// Element i of a 16-byte vector, and the maximum of a vector's elements.
template <bool F32>
__device__ __forceinline__ float element(const uint4& q, int i) {
    const uint32_t* w = &q.x;
    if constexpr (F32) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
}
template <bool F32>
__device__ __forceinline__ float2 pair_of(const uint4& q, int i) { return make_float2(element<F32>(q, i), element<F32>(q, i + 1)); }
template <bool F32>
__device__ __forceinline__ float max_of(const uint4& q) {
    float m = element<F32>(q, 0);
#pragma unroll
    for (int i = 1; i < (F32 ? 4 : 8); ++i) m = max_nan(m, element<F32>(q, i));
    return m;
}

// ---- the kernel ----
// A cluster of C CTAs (one CTA for most vocabularies) takes a row, a slice each, and keeps it in shared memory between the
// statistics and the gradient: the row crosses HBM once in each direction.  One bulk copy brings a slice, started by
// whichever warp is the last to be done with the row before, so that no warp waits to start it.  Three CTAs share an SM: the
// copy and the exchange of statistics of one run beside the arithmetic of the others.  The warps of a row wait for one
// another only for that exchange: each publishes its statistics (to all CTAs of the cluster), then every warp merges all of
// them.
//
// What bounds it: HBM, with the arithmetic close behind (per element of a bf16 row 13 issue slots and 2 special-function
// operations, 57 % and 69 % of what the SMs have while the row streams): loss and gradient over 16384 x 32768 bf16 in 376 to
// 388 us, 0.86 to 0.88 of the copy rate; over 8192 x 131072, four CTAs per row, 763 us, 0.87.  Tried and not kept: the slice in registers
// (2 CTAs per SM, 438 us for the loss over 4096 x 131072 against 398), chunks that are refilled one by one (441 us: the
// waits cost more than the earlier copies gain), a share of the exponentials as polynomials on the FMA pipes (425 us).
// Rows are dealt out in advance (no counter that calls would have to share): the k-th row that is read goes to cluster
// k mod clusters, so that prompt tokens, which cost next to nothing, do not leave some clusters with more work than others.
// Each CTA makes a bit mask of the rows that are read for that, if the batch is neither so small that every cluster has one
// row nor larger than the mask; otherwise row i goes to cluster i mod clusters (1000 x 100003 with a quarter of the rows
// ignored: 73 us with the mask, 78 without; 8000 x 40000: the same).
struct RowsLayout {
    int32_t C;              // CTAs per row
    int32_t stages;         // slices that shared memory holds: one is worked on, copies of later rows go to the others
    int32_t mask_words;     // 32-row words of the mask, 0 = none
    int64_t slice;          // elements per CTA (whole vectors)
};
constexpr int VR_STAGES = 4, VR_RING = 8;       // most stages; row numbers known ahead (a power of two above VR_STAGES)

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void send_stats(uint32_t dst, uint32_t bar, float m, float s, float u, float z) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst),
                 "r"(__float_as_uint(m)), "r"(__float_as_uint(s)), "r"(__float_as_uint(u)), "r"(__float_as_uint(z)), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void bulk_prefetch(const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes));
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Whether a row's logits are needed: it has a valid target, and its loss (a token of weight 0 contributes nothing) or an
// output of its own is wanted.
__device__ __forceinline__ bool row_read(const VocabRows& a, int32_t target, float weight) {
    return (target >= 0) & (target < a.V) & ((a.logp != nullptr) | (a.entropy != nullptr) | (weight != 0.f));
}

// Statistics of a warp's part of a row.  `done` is called when the slice has been read once; `again`: where it is read a second
// time if it has to be (without a gradient its place in shared memory has been given up by then: from L2).
struct WarpStats {
    float m, s, u;          // the reference that the sums are relative to (-inf: no finite logit, sums of 0), sum 2^t, sum t 2^t
};
template <bool F32, bool ENTROPY, int NT, typename Done>
__device__ __forceinline__ WarpStats warp_statistics(const uint4* slice, const uint4* again, int nvec, float zt, int tid, float k2, Done done) {
    constexpr int N = Vec<F32>::N;
    WarpStats r;
    // Sums relative to a reference that any element near the maximum gives as well: the maximum of each thread's first
    // vector.  Finding the true one first would take as many instructions as the sums.
    r.m = warp_max(tid < nvec ? max_nan(zt, max_of<F32>(slice[tid])) : zt);
    // All masked there (-inf): the next vectors in which any lane finds something else; a warp that finds nothing has sums of 0.
    // (4096 x 131072 with all but the 50 largest masked: log-probabilities 246 us, 436 if such warps go through a second time,
    // 203 without a mask.)  The one warp of a short row goes through a second time instead: the look costs it 4 % of a row.
    if (NT > 32 && __builtin_expect(r.m == -INFINITY, 0)) {
#pragma unroll 1
        for (int v = tid + NT; r.m == -INFINITY && v - (tid & 31) < nvec; v += NT) {
            const float x = v < nvec ? max_of<F32>(slice[v]) : -INFINITY;
            if (__any_sync(0xffffffffu, x != -INFINITY)) r.m = warp_max(x);
        }
    }
    {
        const float mr = ref_of(r.m), tt = exponent(zt, mr, k2);
        float2 s2 = make_float2(ex2(tt), 0.f), u2 = make_float2(__fmul_rn(s2.x, tt), 0.f);
#pragma unroll 4
        for (int v = tid; v < nvec; v += NT) {
            const uint4 q = slice[v];
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                float2 t = __fmul2_rn(__fadd2_rn(pair_of<F32>(q, j), make_float2(-mr, -mr)), make_float2(k2, k2));
                if (ENTROPY) t = make_float2(max_nan(t.x, -200.f), max_nan(t.y, -200.f));
                const float2 e = make_float2(ex2(t.x), ex2(t.y));
                s2 = __fadd2_rn(s2, e);
                if (ENTROPY) u2 = __ffma2_rn(e, t, u2);
            }
        }
        done();
        r.s = warp_sum(s2.x + s2.y);
        r.u = ENTROPY ? warp_sum(u2.x + u2.y) : 0.f;
    }
    // again from the true maximum if the reference was too far below it, or if there is a NaN (a sum with a reference among its
    // elements is 1 at least: 0 means that nothing was found)
    if (NT == 32 ? r.m == -INFINITY || !(r.s > 0x1p-30f && r.s < 0x1p40f) : !(r.s == 0.f || (r.s > 0x1p-30f && r.s < 0x1p40f))) {
        r.m = zt;
        for (int v = tid; v < nvec; v += NT) r.m = max_nan(r.m, max_of<F32>(again[v]));
        r.m = warp_max(r.m);
        const float mr = ref_of(r.m), tt = exponent(zt, mr, k2);
        float s = ex2(tt), u = __fmul_rn(s, tt);
        for (int v = tid; v < nvec; v += NT) {
            const uint4 q = again[v];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = exponent(element<F32>(q, j), mr, k2), e = ex2(t);
                s += e;
                u = fmaf(e, t, u);
            }
        }
        r.s = warp_sum(s);
        if (ENTROPY) r.u = warp_sum(u);
    }
    return r;
}

template <bool F32, bool GRAD, bool ENTROPY, bool ENTROPY_GRAD, int NT, bool CLUSTER>
__global__ void __launch_bounds__(NT, 768 / NT) k_vocab_rows(const VocabRows a, const RowsLayout lay) {
    using X = Vec<F32>;
    constexpr int E = F32 ? 4 : 2, W = NT / 32, PARTS = CLUSTER ? 8 * W : W;
    extern __shared__ __align__(128) uint4 s_dynamic[];     // the slices, then the mask
    __shared__ __align__(16) float4 s_part[2][PARTS];       // statistics of all warps of a row
    __shared__ __align__(8) uint64_t s_full[VR_STAGES], s_stat[2];
    __shared__ int64_t s_row[VR_RING];                      // the rows this cluster reads, in order; -1 = no more
    __shared__ int s_done[VR_STAGES], s_copies[VR_STAGES], s_abort;     // warps done with a slice; copies started; given up
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = CLUSTER ? dk_cluster_ctarank() : 0;
    const int C = CLUSTER ? lay.C : 1, stages = lay.stages;
    const int64_t clusters = gridDim.x / C, me = blockIdx.x / C;
    const uint32_t bar_full = smem_u32(s_full), bar_stat = smem_u32(s_stat);
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(bar_full + 8 * i, 1);
            s_done[i] = s_copies[i] = 0;
        }
        mbar_init(bar_stat, 1);
        mbar_init(bar_stat + 8, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // this CTA's part of every row: whole vectors, and behind the last of the row up to 7 elements
    const int64_t V = a.V, begin = min((int64_t)rank * lay.slice, V);
    const int64_t end = (int)rank == C - 1 ? V : min(begin + lay.slice, V);
    const int nvec = (int)((end - begin) / X::N), ntail = (int)(end - begin) - nvec * X::N;
    const int64_t tail = begin + (int64_t)nvec * X::N;
    const int stage_vecs = (int)(lay.slice / X::N);
    // (through a shuffle: a value of each lane's own, which two-element instructions take as it is, not a uniform one)
    const float k2 = __shfl_sync(0xffffffffu, a.inv_temperature * VR_LOG2E, 0);
    auto reads = [&](int64_t row) {
        return row < a.T && row_read(a, a.targets[row], a.terms ? a.weight[row] : 1.f);
    };
    uint32_t* s_mask = reinterpret_cast<uint32_t*>(s_dynamic + (size_t)stages * stage_vecs);
    for (int w0 = warp * 8; w0 < lay.mask_words; w0 += W * 8) {         // eight words' loads at once
        int32_t t[8];
        float wt[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t r = (int64_t)(w0 + k) * 32 + lane;
            t[k] = r < a.T ? a.targets[r] : -1;
            wt[k] = a.terms && r < a.T ? a.weight[r] : 1.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t word = __ballot_sync(0xffffffffu, row_read(a, t[k], wt[k]));
            if (lane == 0 && w0 + k < lay.mask_words) s_mask[w0 + k] = word;
        }
    }
    __syncthreads();
    if (CLUSTER) dk_cluster_sync();
    if (a.terms) dk_launch_dependents();        // the kernel that sums the terms; it waits for this one's end
    auto source = [&](int64_t row) { return (const char*)a.logits + ((size_t)row * a.ld + begin) * E; };
    auto copy = [&](int64_t row, int stage) {            // one thread; the stage is free
        ++s_copies[stage];
        mbar_expect_tx(bar_full + 8 * stage, (uint32_t)nvec * 16);
        bulk_load(smem_u32(s_dynamic + (size_t)stage * stage_vecs), source(row), (uint32_t)nvec * 16, bar_full + 8 * stage);
    };
    // Warp 0 finds the rows.  With a mask: `skip` rows that are read lie before the next one from word `at` on (in which
    // `bits` are left); without: from row `at` on in steps of `clusters`.
    int64_t at = lay.mask_words ? 0 : me, skip = me;
    uint32_t bits = lay.mask_words ? s_mask[0] : 0u;
    auto next_row = [&]() -> int64_t {
        if (lay.mask_words) {
            if (__popc(bits) <= skip) {
                skip -= __popc(bits);
                int64_t w0 = at + 1;
                while (true) {      // 32 words at a time
                    if (w0 >= lay.mask_words) {
                        at = lay.mask_words;
                        bits = 0;
                        skip = 0;
                        return -1;
                    }
                    const uint32_t word = w0 + lane < lay.mask_words ? s_mask[w0 + lane] : 0u;
                    int upto = __popc(word);
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int x = __shfl_up_sync(0xffffffffu, upto, o);
                        if (lane >= o) upto += x;
                    }
                    const uint32_t reached = __ballot_sync(0xffffffffu, upto > skip);
                    if (reached) {
                        const int l = __ffs(reached) - 1;
                        bits = __shfl_sync(0xffffffffu, word, l);
                        skip -= __shfl_sync(0xffffffffu, upto, l) - __popc(bits);
                        at = w0 + l;
                        break;
                    }
                    skip -= __shfl_sync(0xffffffffu, upto, 31);
                    w0 += 32;
                }
            }
            for (; skip > 0; --skip) bits &= bits - 1;
            const int64_t row = at * 32 + __ffs(bits) - 1;
            bits &= bits - 1;
            skip = clusters - 1;
            return row;
        }
        while (at < a.T) {
            const uint32_t found = __ballot_sync(0xffffffffu, reads(at + lane * clusters));
            if (found) {
                const int64_t row = at + (int64_t)(__ffs(found) - 1) * clusters;
                at = row + clusters;
                return row;
            }
            at += 32 * clusters;
        }
        return -1;
    };
    if (warp == 0) {
        bool more = true;
        for (int i = 0; i < stages; ++i) {
            const int64_t row = more ? next_row() : -1;
            more = row >= 0;
            if (lane == 0) {
                s_row[i] = row;
                if (more && nvec > 0) copy(row, i);
            }
        }
    }
    // rows that are not read, row i by cluster i mod clusters, while the first copies are under way
    for (int64_t r0 = me; r0 < a.T; r0 += 32 * clusters) {
        uint32_t left = __ballot_sync(0xffffffffu, r0 + lane * clusters < a.T && !reads(r0 + lane * clusters));
        for (; left; left &= left - 1) {
            const int64_t row = r0 + (int64_t)(__ffs(left) - 1) * clusters;
            if (rank == 0 && tid == 0) {
                if (a.targets[row] >= V) dk_report(a.status, DEV_BAD_INDEX, (int)row);
                if (a.logp) a.logp[row] = 0.f;
                if (a.entropy) a.entropy[row] = 0.f;
                if (a.terms) a.terms[row] = PolicyTerms{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            }
            if (GRAD) {
                char* dzr = (char*)a.dlogits + (size_t)row * a.lddl * E;
                uint4* dz = reinterpret_cast<uint4*>(dzr + begin * E);
                for (int v = tid; v < nvec; v += NT) __stcs(dz + v, make_uint4(0, 0, 0, 0));
                if (tid < ntail) X::store(dzr, tail + tid, 0.f);
            }
        }
    }
    __syncthreads();        // s_row
    TokenIn in = {0.f, 0.f, 0.f, 1.f};
    uint32_t phase = 0;
    for (int it = 0, stage = 0; s_row[it & (VR_RING - 1)] >= 0; ++it) {
        const int64_t row = s_row[it & (VR_RING - 1)];
        const bool first = rank == 0 && tid == 0;
        const int32_t target = a.targets[row];
        if (a.terms) {
            in.w = a.weight[row];
            in.old = a.old_logp[row];
            in.A = a.adv[row];
            if (a.ref_logp) in.ref = a.ref_logp[row];
        }
        const char* z = (const char*)a.logits + (size_t)row * a.ld * E;
        const uint4* s_slice = s_dynamic + (size_t)stage * stage_vecs;
        if (warp == 0) {
            const int64_t later = s_row[(it + stages - 1) & (VR_RING - 1)] >= 0 ? next_row() : -1;
            if (lane == 0) s_row[(it + stages) & (VR_RING - 1)] = later;
        }
        // a warp is done with the slice: the last one starts the copy of a later row's
        auto release = [&]() {
            __syncwarp();
            if (lane == 0) {
                __threadfence_block();
                if (atomicAdd(&s_done[stage], 1) == W - 1) {
                    s_done[stage] = 0;
                    __threadfence_block();
                    const int64_t later = s_row[(it + stages) & (VR_RING - 1)];
                    if (nvec > 0 && later >= 0 && s_abort == 0) copy(later, stage);
                }
            }
        };
        RowGrad g = {0.f, 0.f, 0.f};
        float m = 0.f, log2s = 0.f, za = 0.f, zt = -INFINITY;      // za: the target's logit
        if (tid < ntail) zt = X::load(z, tail + tid);
        if (rank == 0 && warp == 0) za = X::load(z, target);
        if (nvec > 0 && !__all_sync(0xffffffffu, mbar_wait(bar_full + 8 * stage, phase, &s_abort, 2))) break;
        const uint4* again = GRAD ? s_slice : reinterpret_cast<const uint4*>(z + begin * E);
        const WarpStats ws = warp_statistics<F32, ENTROPY, NT>(s_slice, again, nvec, zt, tid, k2, [&]() {
            if (!GRAD) release();
        });
        // Two buffers: a warp writes for row i + 2 only after all warps have written for row i + 1, which they do
        // when they have read row i.
        const int b = it & 1;
        if (CLUSTER) {
            if (tid == 0) mbar_expect_tx(bar_stat + 8 * b, (uint32_t)(C * W * 16));
            if (lane < C)
                send_stats(dk_map_to_cta(smem_u32(&s_part[b][rank * W + warp]), lane), dk_map_to_cta(bar_stat + 8 * b, lane), ws.m,
                           ws.s, ws.u, za);
            if (!__all_sync(0xffffffffu, mbar_wait(bar_stat + 8 * b, (it >> 1) & 1, &s_abort, 3))) break;
        } else if (PARTS > 1) {
            if (lane == 0) s_part[b][warp] = make_float4(ws.m, ws.s, ws.u, za);
            __syncthreads();
        }
        // the next row into L2 while this one's gradient leaves (not earlier: the rows in flight and what has been
        // written of the gradient fill the part of L2 that would have to keep it)
        if (GRAD && tid == 0 && nvec > 0 && stages == 1 && s_row[(it + 1) & (VR_RING - 1)] >= 0)
            bulk_prefetch(source(s_row[(it + 1) & (VR_RING - 1)]), (uint32_t)nvec * 16);
        // all warps' statistics, relative to the row's maximum; up to PARTS / 32 of them per lane
        float rs = 0.f, ru = 0.f;
        if (PARTS == 1) {
            m = ref_of(ws.m);
            rs = ws.s;
            ru = ws.u;
        } else {
            constexpr int PER = (PARTS + 31) / 32;
            float4 x[PER];
            float rm = -INFINITY;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                x[i] = lane + 32 * i < C * W ? s_part[b][lane + 32 * i] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
                rm = max_nan(rm, x[i].x);
            }
            m = ref_of(warp_max(rm));
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float d = exponent(x[i].x, m, k2), f = ex2(d);
                rs = fmaf(f, x[i].y, rs);
                if (ENTROPY) ru = fmaf(f, fmaf(x[i].y, d, x[i].z), ru);
            }
            rs = warp_sum(rs);
            if (ENTROPY) ru = warp_sum(ru);
            za = s_part[b][0].w;
        }
        const bool dist = !(rs == 0.f);        // else there is no finite logit
        log2s = dist ? lg2(rs) : 0.f;
        const float logp = dist ? fmaf(za - m, k2, -log2s) * VR_LN2 : 0.f;
        const float H = ENTROPY && dist ? (log2s - __fdividef(ru, rs)) * VR_LN2 : 0.f;
        if (first) {
            if (a.logp) a.logp[row] = logp;
            if (a.entropy) a.entropy[row] = H;
        }
        const bool live = dist && in.w != 0.f;
        if (a.terms && live) {
            PolicyTerms t;
            g = token_terms(a, in, logp, H, log2s, &t);
            if (first) a.terms[row] = t;
        }
        if (a.terms && !live && first) a.terms[row] = PolicyTerms{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (GRAD) {
            char* dzr = (char*)a.dlogits + (size_t)row * a.lddl * E;
            uint4* dz = reinterpret_cast<uint4*>(dzr + begin * E);
            if (live) {
#pragma unroll 4
                for (int v = tid; v < nvec; v += NT) {
                    const uint4 q = s_slice[v];
                    float2 f[X::N / 2];
#pragma unroll
                    for (int j = 0; j < X::N; j += 2) {
                        const float2 d = __fadd2_rn(pair_of<F32>(q, j), make_float2(-m, -m));
                        if (ENTROPY_GRAD) {
                            float2 t = __fmul2_rn(d, make_float2(k2, k2));
                            t = make_float2(max_nan(t.x, -200.f), max_nan(t.y, -200.f));
                            const float2 w = __fadd2_rn(t, make_float2(-log2s, -log2s));
                            f[j / 2] = __fmul2_rn(make_float2(ex2(w.x), ex2(w.y)), __ffma2_rn(make_float2(g.alpha, g.alpha), t, make_float2(g.beta, g.beta)));
                        } else {
                            const float2 w = __ffma2_rn(d, make_float2(k2, k2), make_float2(-log2s, -log2s));
                            f[j / 2] = __fmul2_rn(make_float2(ex2(w.x), ex2(w.y)), make_float2(g.beta, g.beta));
                        }
                    }
                    __stcs(dz + v, X::pack(f));
                }
                // the target's element once more, by the thread that has just written its vector
                if (target >= begin && target < tail && tid == (int)((target - begin) / X::N) % NT) {
                    const float t = exponent(za, m, k2);
                    X::store(dzr, target, ex2(t - log2s) * fmaf(g.alpha, t, g.beta) + g.gamma);
                }
            } else {
                for (int v = tid; v < nvec; v += NT) __stcs(dz + v, make_uint4(0, 0, 0, 0));
            }
            release();
            if (tid < ntail) {
                float o = 0.f;
                if (live) {
                    const float t = exponent(zt, m, k2);
                    o = ex2(t - log2s) * fmaf(g.alpha, t, g.beta) + (tail + tid == target ? g.gamma : 0.f);
                }
                X::store(dzr, tail + tid, o);
            }
        }
        if (++stage == stages) {
            stage = 0;
            phase ^= 1;
        }
    }
    __syncthreads();
    if (s_abort != 0 && tid == 0) {
        // given up: the shared memory is left only when no copy into it is in flight
        dk_report(a.status, DEV_TIMEOUT, s_abort * 1000000 + (int)blockIdx.x);
        const unsigned long long t0 = global_ns();
        for (int i = 0; i < stages; ++i)
            while (s_copies[i] > 0 && !mbar_try_wait(bar_full + 8 * i, (s_copies[i] - 1) & 1) && global_ns() - t0 < WAIT_LIMIT_NS) {}
    }
    if (CLUSTER) {
        // no CTA of a cluster leaves while another may still write to its shared memory
        __syncwarp();
        dk_cluster_sync();
    }
}

template <bool F32, bool GRAD, bool ENTROPY, bool ENTROPY_GRAD, int NT, bool CLUSTER>
static marlaas_status_t launch_rows(const marlaas_pool* pool, const VocabRows& r, int C, cudaStream_t st) {
    constexpr int N = F32 ? 4 : 8, SIZES = 18;
    auto kernel = k_vocab_rows<F32, GRAD, ENTROPY, ENTROPY_GRAD, NT, CLUSTER>;
    RowsLayout lay;
    lay.C = C;
    lay.slice = cdiv(cdiv(r.V, C), N) * N;
    // as many stages as leave the SM room for 768 threads; the mask where a CTA's 8 warps make it in a few microseconds (with
    // shorter rows there are more of them per CTA, which evens them out, and fewer warps to make it)
    const int64_t slice_bytes = lay.slice * (F32 ? 4 : 2), words = cdiv(r.T, 32);
    const int64_t mask_bytes = NT >= 256 && words <= 256 ? words * 4 : 0;
    lay.stages = (int)std::max<int64_t>(1, std::min<int64_t>(VR_STAGES, (NT * 280 - mask_bytes) / slice_bytes));
    // shared memory in sixteenths of the largest slice (128 KB for 256 threads), so that the number of rows the device holds
    // is asked for once per device and size
    const int64_t unit = (int64_t)NT * 32;
    const int size = (int)cdiv(lay.stages * slice_bytes + mask_bytes, unit);
    const size_t smem = (size_t)size * unit;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = CLUSTER ? 1 : 0;
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.gridDim = dim3(C);
    static std::atomic<int> resident[MAX_DEVICES][9][SIZES];
    std::atomic<int>* known = pool->device < MAX_DEVICES && size < SIZES ? &resident[pool->device][C][size] : nullptr;
    int rows = known ? known->load(std::memory_order_relaxed) : 0;
    if (rows == 0) {
        MARLAAS_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)((SIZES - 1) * unit)));
        if (CLUSTER) {
            MARLAAS_CUDA_TRY(cudaOccupancyMaxActiveClusters(&rows, kernel, &cfg));
        } else {
            MARLAAS_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&rows, kernel, NT, smem));
            rows *= pool->sm_count;
        }
        if (rows < 1) return fail(MARLAAS_ERR_CUDA, "k_vocab_rows: no room for a cluster of %d", C);
        if (known) known->store(rows, std::memory_order_relaxed);
    }
    lay.mask_words = r.T > rows && mask_bytes ? (int)words : 0;
    cfg.gridDim = dim3((unsigned)(std::min<int64_t>(rows, r.T) * C));
    MARLAAS_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, r, lay));
    MARLAAS_LAUNCH_CHECK("k_vocab_rows");
    return MARLAAS_OK;
}

// The shape of a launch, from the sizes alone (not from what is wanted of the rows, so that all calls on a batch sum in one
// order; and products and sums are fused where the code says so, not as the compiler likes): the log-probabilities of
// marlaas_token_logprobs and of the loss are the same bits, and the ratios of an update's first pass exactly 1.
template <bool F32, bool GRAD, bool ENTROPY, bool ENTROPY_GRAD>
static marlaas_status_t launch_shape(const marlaas_pool* pool, const VocabRows& r, cudaStream_t st) {
    const int64_t vecs = cdiv(r.V, F32 ? 4 : 8);
    // as few CTAs per row as their shared memory allows
    constexpr int BIG = 256;
    int C = (int)std::min<int64_t>(8, cdiv(vecs * 16, BIG * 280));
    // few rows: more CTAs for each, down to one vector per thread (1 to 4 rows of 131072: 7.7 us against 8.7; from 16 rows of
    // 131072 or 32 of 32768 on it is even or slower: 9.5 against 8.9)
    while (C < 8 && r.T * C * 8 <= pool->sm_count && vecs > (int64_t)C * BIG) C = std::min(8, 2 * C);
    if (C > 1) return launch_rows<F32, GRAD, ENTROPY, ENTROPY_GRAD, BIG, true>(pool, r, C, st);
    // Shorter rows: as few warps as hold 16 vectors per thread, since part of a row's work is every warp's (20000 x 4000: 82 us
    // with one warp, 97 with two; 10000 x 8000: 73 with two, 80 with four; 8000 x 16000: 100 with four, 120 with eight).
    if (vecs <= 32 * 16) return launch_rows<F32, GRAD, ENTROPY, ENTROPY_GRAD, 32, false>(pool, r, 1, st);
    if (vecs <= 64 * 16) return launch_rows<F32, GRAD, ENTROPY, ENTROPY_GRAD, 64, false>(pool, r, 1, st);
    if (vecs <= 128 * 16) return launch_rows<F32, GRAD, ENTROPY, ENTROPY_GRAD, 128, false>(pool, r, 1, st);
    return launch_rows<F32, GRAD, ENTROPY, ENTROPY_GRAD, BIG, false>(pool, r, 1, st);
}

marlaas_status_t launch_vocab_rows(const marlaas_pool* pool, const VocabRows& r, cudaStream_t st) {
    const bool entropy = r.entropy || r.terms, eg = r.dlogits && r.entropy_coef != 0.f;
    if (r.f32) return !r.dlogits ? (entropy ? launch_shape<true, false, true, false>(pool, r, st) : launch_shape<true, false, false, false>(pool, r, st))
                                 : eg ? launch_shape<true, true, true, true>(pool, r, st) : launch_shape<true, true, true, false>(pool, r, st);
    return !r.dlogits ? (entropy ? launch_shape<false, false, true, false>(pool, r, st) : launch_shape<false, false, false, false>(pool, r, st))
                      : eg ? launch_shape<false, true, true, true>(pool, r, st) : launch_shape<false, true, true, false>(pool, r, st);
}

}  // namespace marlaas
