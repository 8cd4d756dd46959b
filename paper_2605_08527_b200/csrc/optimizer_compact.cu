// AdamW and commit with both moments in 8 bits (Algorithm 1: "PolicyUpdate" and the commit of the new adapter version;
// Methods, Multi-Task Manager: per-task optimizer state, which at 8 bytes per element is four times the bf16 adapter
// itself).  The state's format is in marlaas.h.  Per element: gradient 4 B read, master 4 + 4, moments 2.06 + 2.06, the
// pool's bf16 2 written = 18.1 bytes and no reuse: bound by HBM.
#include <string.h>

#include <cmath>
#include <numeric>

#include "internal.cuh"

namespace marlaas {

constexpr int OC_THREADS = 256;
constexpr int OC_BLOCK = 256;               // elements that share their exponents: one warp, 8 per lane
constexpr int OC_STATE_BYTES = 528;
constexpr int OC_UNIT = 2048;               // elements of B (and at least, of A) per CTA
constexpr int OC_MAX_TENANTS = 256;         // tenants per launch
constexpr uint32_t OC_M_ORDERS = 15, OC_V_ORDERS = 31;      // binary orders below the block's largest exponent

struct CompactTenant {
    const float* dA;
    const float* dB;
    float* A;
    float* B;
    uint8_t* sA;
    uint8_t* sB;
    uint64_t id;
    int32_t slot;
    uint16_t rank, vec;     // vec: gradients and masters are 16-byte aligned
};
// The table of a launch; three sizes, so that a few tenants do not pay for the parameters of 256.
template <int N>
struct CompactArgs {
    int n, P, RP, cap;
    int64_t K, ldB;
    int64_t part_begin[MARLAAS_MAX_PARTS + 1];
    float lr, b1, b2, one_b1, one_b2, eps, wd, gscale, c1, c2;
    uint64_t seed, step;
    bf16* At;
    bf16* Bs;
    int32_t first[2 * N + 1];       // first CTA of tenant t's A (2t) and B (2t + 1)
    CompactTenant t[N];
};

// Random bits of an element: two rounds of xor-shift and multiplication by odd constants (2^32 divided by the golden ratio,
// and by the square root of 2), a bijection of the 32-bit numbers.
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x9E3779B9u;
    x = (x ^ (x >> 15)) * 0xB504F333u;
    return x ^ (x >> 16);
}
__device__ __forceinline__ uint32_t stream_key(uint64_t seed, uint64_t step, uint64_t tenant, uint32_t matrix) {
    const uint32_t w[7] = {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32),
                           (uint32_t)tenant, (uint32_t)(tenant >> 32), matrix};
    uint32_t k = 0;
#pragma unroll
    for (int i = 0; i < 7; ++i) k = mix32((k + 0x9E3779B9u) ^ w[i]);
    return k;
}

// Codes count in steps of 2^20 of the fp32 bit pattern (sign cut off): exponent and 3 mantissa bits.
__device__ __forceinline__ uint32_t code_base(uint32_t E, uint32_t orders) { return E > orders ? (E - orders) * 8 : 0; }
__device__ __forceinline__ float code_value(uint32_t c, uint32_t base) { return c ? __uint_as_float((c + base) << 20) : 0.f; }
// The magnitude to store: not finite -> 0; never so large that rounding up leaves the finite numbers.
__device__ __forceinline__ uint32_t magnitude(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b >= 0x7f800000u ? 0u : min(b, 0x7f700000u);
}
// The exponent that holds a block's largest magnitude also after rounding up.
__device__ __forceinline__ uint32_t block_exponent(uint32_t largest) { return (largest + 0xfffffu) >> 23; }
__device__ __forceinline__ int32_t code_of(uint32_t mag, uint32_t rnd16, uint32_t base) { return (int32_t)((mag + (rnd16 << 4)) >> 20) - (int32_t)base; }

struct CompactHyper {
    float lr, b1, b2, one_b1, one_b2, eps, wd, gscale, c1, c2;
};

// Elements [first, first + 256) of a matrix of n elements: lane's elements are 4 lane .. 4 lane + 3 and 128 further on.
// Writes masters and state, leaves the new masters in th[8].
__device__ __forceinline__ void compact_block(const CompactHyper& h, const float* __restrict__ grad, float* __restrict__ theta,
                                              uint8_t* __restrict__ state, int64_t first, int64_t n, bool vec, uint32_t key,
                                              int lane, float (&th)[8]) {
    uint8_t* blk = state + (first / OC_BLOCK) * OC_STATE_BYTES;
    float g[8];
    uint32_t mc[2], vc[2];
    bool in[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int64_t e = first + 128 * q + 4 * lane;
        in[q] = e < n;      // n is a multiple of 8
        mc[q] = vc[q] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) g[4 * q + i] = th[4 * q + i] = 0.f;
        if (in[q]) {
            mc[q] = reinterpret_cast<const uint32_t*>(blk)[32 * q + lane];
            vc[q] = reinterpret_cast<const uint32_t*>(blk + 256)[32 * q + lane];
            if (vec) {
                const float4 a = __ldcs(reinterpret_cast<const float4*>(grad + e)), b = *reinterpret_cast<const float4*>(theta + e);
                g[4 * q] = a.x; g[4 * q + 1] = a.y; g[4 * q + 2] = a.z; g[4 * q + 3] = a.w;
                th[4 * q] = b.x; th[4 * q + 1] = b.y; th[4 * q + 2] = b.z; th[4 * q + 3] = b.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    g[4 * q + i] = grad[e + i];
                    th[4 * q + i] = theta[e + i];
                }
            }
        }
    }
    const uint32_t E = *reinterpret_cast<const uint16_t*>(blk + 512);
    const uint32_t bm = code_base(E & 255u, OC_M_ORDERS), bv = code_base(E >> 8, OC_V_ORDERS);
    uint32_t am[8], av[8], neg = 0, top_m = 0, top_v = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t cm = (mc[i >> 2] >> (8 * (i & 3))) & 255u, cv = (vc[i >> 2] >> (8 * (i & 3))) & 255u;
        float m = code_value(cm & 127u, bm);
        m = (cm & 128u) ? -m : m;
        float v = code_value(cv, bv);
        const float gr = __fmul_rn(h.gscale, g[i]);
        // separate roundings of products and sums: the same bits wherever this is computed
        m = __fadd_rn(__fmul_rn(h.b1, m), __fmul_rn(h.one_b1, gr));
        v = __fadd_rn(__fmul_rn(h.b2, v), __fmul_rn(__fmul_rn(h.one_b2, gr), gr));
        const float mh = m * h.c1, vh = v * h.c2;
        th[i] -= h.lr * (mh / (sqrtf(vh) + h.eps) + h.wd * th[i]);
        am[i] = magnitude(m);
        av[i] = magnitude(v);
        neg |= (uint32_t)(m < 0.f) << i;
        top_m = max(top_m, am[i]);
        top_v = max(top_v, av[i]);
    }
    top_m = __reduce_max_sync(0xffffffffu, top_m);
    top_v = __reduce_max_sync(0xffffffffu, top_v);
    const uint32_t Em = block_exponent(top_m), Ev = block_exponent(top_v);
    const uint32_t nm = code_base(Em, OC_M_ORDERS), nv = code_base(Ev, OC_V_ORDERS);
    mc[0] = mc[1] = vc[0] = vc[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = mix32((uint32_t)first + (uint32_t)(128 * (i >> 2) + 4 * lane + (i & 3)) + key);
        const uint32_t cm = (uint32_t)max(code_of(am[i], r & 0xffffu, nm), 0) | (((neg >> i) & 1u) << 7);
        const uint32_t cv = av[i] ? (uint32_t)max(code_of(av[i], r >> 16, nv), 1) : 0u;
        mc[i >> 2] |= cm << (8 * (i & 3));
        vc[i >> 2] |= cv << (8 * (i & 3));
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        reinterpret_cast<uint32_t*>(blk)[32 * q + lane] = mc[q];
        reinterpret_cast<uint32_t*>(blk + 256)[32 * q + lane] = vc[q];
        if (in[q]) {
            const int64_t e = first + 128 * q + 4 * lane;
            if (vec) {
                *reinterpret_cast<float4*>(theta + e) = make_float4(th[4 * q], th[4 * q + 1], th[4 * q + 2], th[4 * q + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) theta[e + i] = th[4 * q + i];
            }
        }
    }
    if (lane == 0) *reinterpret_cast<uint16_t*>(blk + 512) = (uint16_t)(Em | (Ev << 8));
}

// Rows of A per CTA: whole state blocks, at least 64 rows (128-byte runs of the pool's At rows) and OC_UNIT elements.
__host__ __device__ __forceinline__ int rows_per_cta(int r) {
    int g = r, b = OC_BLOCK;        // 256 / gcd(256, r) rows are whole blocks
    while (b) {
        const int c = g % b;
        g = b;
        b = c;
    }
    const int step = OC_BLOCK / g, want = max(64, (OC_UNIT + r - 1) / r);
    return (want + step - 1) / step * step;
}
__host__ __device__ __forceinline__ int tile_pitch(int r) { return r | 1; }     // odd: column reads spread over the banks

__device__ __forceinline__ int64_t state_bytes(int64_t n) { return (n + OC_BLOCK - 1) / OC_BLOCK * OC_STATE_BYTES; }

// One CTA per unit: a run of B, stored as the pool stores it, or a tile of rows of A, which goes through shared memory so
// that both the reads of A [K][r] and the writes of the pool's At rows [r][K] are contiguous.
template <int N>
__global__ void __launch_bounds__(OC_THREADS) k_adamw_compact(const __grid_constant__ CompactArgs<N> a) {
    extern __shared__ bf16 tile[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int lo = 0, hi = 2 * a.n;       // the last entry whose first CTA is not after this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= (int)blockIdx.x) lo = mid; else hi = mid;
    }
    const CompactTenant& t = a.t[lo >> 1];
    const int r = t.rank;
    const bool is_b = lo & 1, vec = t.vec != 0;
    int u = (int)blockIdx.x - a.first[lo];
    const CompactHyper h = {a.lr, a.b1, a.b2, a.one_b1, a.one_b2, a.eps, a.wd, a.gscale, a.c1, a.c2};
    if (is_b) {
        int p = 0;
        int64_t soff = 0;
        for (; p < a.P - 1; ++p) {
            const int64_t n = (int64_t)r * (a.part_begin[p + 1] - a.part_begin[p]);
            const int units = (int)((n + OC_UNIT - 1) / OC_UNIT);
            if (u < units) break;
            u -= units;
            soff += state_bytes(n);
        }
        const int64_t c0 = a.part_begin[p], Np = a.part_begin[p + 1] - c0, n = (int64_t)r * Np;
        const uint32_t key = stream_key(a.seed, a.step, t.id, 2u * p + 1u);
        const int64_t e0 = (int64_t)u * OC_UNIT + warp * OC_BLOCK;
        if (e0 >= n) return;
        float th[8];
        compact_block(h, t.dB + (int64_t)r * c0, t.B + (int64_t)r * c0, t.sB + soff, e0, n, vec, key, lane, th);
        bf16* bs = a.Bs + (size_t)t.slot * a.RP * a.ldB + c0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t e = e0 + 128 * q + 4 * lane;
            if (e >= n) continue;
            const int64_t j = e / Np;       // four elements of one row: Np is a multiple of 8
            __nv_bfloat162 x = __floats2bfloat162_rn(th[4 * q], th[4 * q + 1]), y = __floats2bfloat162_rn(th[4 * q + 2], th[4 * q + 3]);
            *reinterpret_cast<uint2*>(bs + j * a.ldB + (e - j * Np)) = make_uint2(*reinterpret_cast<uint32_t*>(&x), *reinterpret_cast<uint32_t*>(&y));
        }
        return;
    }
    const int R = rows_per_cta(r), pitch = tile_pitch(r);
    const int per_part = (int)((a.K + R - 1) / R);
    const int p = u / per_part;
    const int64_t k0 = (int64_t)(u - p * per_part) * R, n = a.K * r, poff = (int64_t)p * n;
    const int rows = (int)min((int64_t)R, a.K - k0);
    const uint32_t key = stream_key(a.seed, a.step, t.id, 2u * p);
    for (int b = warp * OC_BLOCK; b < rows * r; b += OC_THREADS / 32 * OC_BLOCK) {
        float th[8];
        compact_block(h, t.dA + poff, t.A + poff, t.sA + p * state_bytes(n), k0 * r + b, n, vec, key, lane, th);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = b + 128 * q + 4 * lane;
            int kk = e / r, j = e - kk * r;
            if (e >= rows * r) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                tile[kk * pitch + j] = __float2bfloat16_rn(th[4 * q + i]);
                if (++j == r) {
                    j = 0;
                    ++kk;
                }
            }
        }
    }
    __syncthreads();
    bf16* at = a.At + ((size_t)p * a.cap + t.slot) * a.RP * (size_t)a.K + k0;
    const int groups = rows / 8;        // K and R are multiples of 8
    for (int x = tid; x < groups * r; x += OC_THREADS) {
        const int j = x / groups, g8 = (x - j * groups) * 8;
        uint4 o;
        uint32_t* w = &o.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 y;
            y.x = tile[(g8 + 2 * i) * pitch + j];
            y.y = tile[(g8 + 2 * i + 1) * pitch + j];
            w[i] = *reinterpret_cast<uint32_t*>(&y);
        }
        *reinterpret_cast<uint4*>(at + (size_t)j * a.K + g8) = o;
    }
}

// One warp per block of a state.
__global__ void __launch_bounds__(OC_THREADS) k_compact_export(const uint8_t* __restrict__ state, float* __restrict__ m,
                                                               float* __restrict__ v, int64_t blocks) {
    const int lane = threadIdx.x & 31;
    const int64_t w = ((int64_t)blockIdx.x * OC_THREADS + threadIdx.x) >> 5, nw = (int64_t)gridDim.x * (OC_THREADS / 32);
    for (int64_t b = w; b < blocks; b += nw) {
        const uint8_t* blk = state + b * OC_STATE_BYTES;
        const uint32_t E = *reinterpret_cast<const uint16_t*>(blk + 512);
        const uint32_t bm = code_base(E & 255u, OC_M_ORDERS), bv = code_base(E >> 8, OC_V_ORDERS);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t mc = reinterpret_cast<const uint32_t*>(blk)[32 * q + lane];
            const uint32_t vc = reinterpret_cast<const uint32_t*>(blk + 256)[32 * q + lane];
            float fm[4], fv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t cm = (mc >> (8 * i)) & 255u;
                fm[i] = code_value(cm & 127u, bm);
                fm[i] = (cm & 128u) ? -fm[i] : fm[i];
                fv[i] = code_value((vc >> (8 * i)) & 255u, bv);
            }
            const int64_t e = b * OC_BLOCK + 128 * q + 4 * lane;
            if (m) *reinterpret_cast<float4*>(m + e) = make_float4(fm[0], fm[1], fm[2], fm[3]);
            if (v) *reinterpret_cast<float4*>(v + e) = make_float4(fv[0], fv[1], fv[2], fv[3]);
        }
    }
}

template <int N>
static marlaas_status_t launch_compact(const marlaas_pool* pool, const CompactTenant* t, int n, const marlaas_adamw_t& hp,
                                       uint64_t seed, cudaStream_t st) {
    CompactArgs<N> a;
    a.n = n; a.P = pool->P; a.RP = pool->RP; a.cap = pool->cap; a.K = pool->K; a.ldB = pool->ldB;
    for (int p = 0; p <= MARLAAS_MAX_PARTS; ++p) a.part_begin[p] = pool->part_begin[p];
    a.lr = hp.lr; a.b1 = hp.beta1; a.b2 = hp.beta2; a.one_b1 = 1.f - hp.beta1; a.one_b2 = 1.f - hp.beta2;
    a.eps = hp.eps; a.wd = hp.weight_decay; a.gscale = hp.grad_scale;
    a.c1 = (float)(1.0 / (1.0 - std::pow((double)hp.beta1, (double)hp.step)));
    a.c2 = (float)(1.0 / (1.0 - std::pow((double)hp.beta2, (double)hp.step)));
    a.seed = seed; a.step = (uint64_t)hp.step;
    a.At = pool->d_At; a.Bs = pool->d_Bs;
    int64_t ctas = 0;
    size_t smem = 0;
    for (int i = 0; i < n; ++i) {
        const int r = t[i].rank, R = rows_per_cta(r);
        a.t[i] = t[i];
        a.first[2 * i] = (int32_t)ctas;
        ctas += (int64_t)pool->P * cdiv(pool->K, R);
        a.first[2 * i + 1] = (int32_t)ctas;
        for (int p = 0; p < pool->P; ++p) ctas += cdiv((int64_t)r * (pool->part_begin[p + 1] - pool->part_begin[p]), OC_UNIT);
        smem = std::max(smem, sizeof(bf16) * (size_t)R * tile_pitch(r));
        if (ctas >= (1ll << 31)) return fail(MARLAAS_ERR_INVALID_ARG, "pool_adamw_compact_commit: too many elements for one call");
    }
    a.first[2 * n] = (int32_t)ctas;
    if (smem > 48 * 1024)
        MARLAAS_CUDA_TRY(cudaFuncSetAttribute(k_adamw_compact<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    k_adamw_compact<N><<<(unsigned)ctas, OC_THREADS, smem, st>>>(a);
    MARLAAS_LAUNCH_CHECK("k_adamw_compact");
    return MARLAAS_OK;
}

}  // namespace marlaas

using namespace marlaas;

extern "C" {

size_t marlaas_adamw_compact_state_bytes(int64_t n) {
    if (n <= 0) return 0;
    return (size_t)cdiv(n, OC_BLOCK) * OC_STATE_BYTES;
}

marlaas_status_t marlaas_adapter_pool_adamw_compact_commit(marlaas_pool_t* pool, int32_t n, const uint64_t* tenant_ids,
                                                           const uint64_t* new_versions, const float* const* dA,
                                                           const float* const* dB, float* const* A, float* const* B,
                                                           void* const* state_A, void* const* state_B,
                                                           const int32_t* ranks, const marlaas_adamw_t* hp,
                                                           uint64_t seed, void* cuda_stream) try {
    const char* fn = "pool_adamw_compact_commit";
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (n < 0) return fail(MARLAAS_ERR_INVALID_ARG, "%s: negative tenant count", fn);
    if (n == 0) return MARLAAS_OK;
    if (!tenant_ids || !dA || !dB || !A || !B || !state_A || !state_B || !hp)
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: a table or the hyper-parameters are NULL", fn);
    if (hp->step < 1) return fail(MARLAAS_ERR_INVALID_ARG, "%s: step %lld < 1", fn, (long long)hp->step);
    if (!(hp->beta1 >= 0.f && hp->beta1 < 1.f && hp->beta2 >= 0.f && hp->beta2 < 1.f))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: beta1, beta2 must lie in [0, 1)", fn);
    std::vector<CompactTenant> t((size_t)n);
    std::vector<char> seen((size_t)pool->cap, 0);
    for (int i = 0; i < n; ++i) {
        int slot = -1;
        for (int s = 0; s < pool->cap; ++s)
            if (pool->slots[s].used && pool->slots[s].tenant_id == tenant_ids[i]) { slot = s; break; }
        const unsigned long long id = (unsigned long long)tenant_ids[i];
        if (slot < 0) return fail(MARLAAS_ERR_UNKNOWN_TENANT, "%s: tenant %llu is not registered", fn, id);
        if (pool->slots[slot].rank <= 0) return fail(MARLAAS_ERR_INVALID_ARG, "%s: tenant %llu has rank 0", fn, id);
        if (ranks && ranks[i] != pool->slots[slot].rank)
            return fail(MARLAAS_ERR_INVALID_ARG, "%s: tenant %llu has rank %d, its buffers are of rank %d", fn, id,
                        (int)pool->slots[slot].rank, (int)ranks[i]);
        if (seen[slot]) return fail(MARLAAS_ERR_INVALID_ARG, "%s: tenant %llu is listed twice", fn, id);
        seen[slot] = 1;
        const void* ps[4] = {dA[i], dB[i], A[i], B[i]};
        uintptr_t low = 0;
        for (const void* q : ps) {
            if (!q || ((uintptr_t)q & 3))
                return fail(MARLAAS_ERR_INVALID_ARG, "%s: tenant %llu: a pointer is NULL or not 4-byte aligned", fn, id);
            low |= (uintptr_t)q;
        }
        if (!state_A[i] || !state_B[i] || (((uintptr_t)state_A[i] | (uintptr_t)state_B[i]) & 15))
            return fail(MARLAAS_ERR_INVALID_ARG, "%s: tenant %llu: a state is NULL or not 16-byte aligned", fn, id);
        t[i] = CompactTenant{dA[i], dB[i], A[i], B[i], (uint8_t*)state_A[i], (uint8_t*)state_B[i], tenant_ids[i], slot,
                             (uint16_t)pool->slots[slot].rank, (uint16_t)((low & 15) == 0)};
    }
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    for (int i0 = 0; i0 < n; i0 += OC_MAX_TENANTS) {
        const int m = std::min(OC_MAX_TENANTS, n - i0);
        marlaas_status_t rc = m <= 8    ? launch_compact<8>(pool, t.data() + i0, m, *hp, seed, (cudaStream_t)cuda_stream)
                              : m <= 48 ? launch_compact<48>(pool, t.data() + i0, m, *hp, seed, (cudaStream_t)cuda_stream)
                                        : launch_compact<OC_MAX_TENANTS>(pool, t.data() + i0, m, *hp, seed, (cudaStream_t)cuda_stream);
        if (rc != MARLAAS_OK) return rc;
    }
    for (int i = 0; i < n; ++i) {
        SlotMeta& m = pool->slots[t[i].slot];
        m.version = new_versions ? new_versions[i] : m.version + 1;
    }
    return MARLAAS_OK;
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "pool_adamw_compact_commit: %s", e.what());
}

marlaas_status_t marlaas_adamw_compact_state_export(marlaas_pool_t* pool, int64_t blocks, const void* state, float* m, float* v,
                                                    void* cuda_stream) {
    const char* fn = "adamw_compact_state_export";
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (blocks < 0) return fail(MARLAAS_ERR_INVALID_ARG, "%s: negative block count", fn);
    if (blocks == 0 || (!m && !v)) return MARLAAS_OK;
    if (!state || (((uintptr_t)state | (uintptr_t)m | (uintptr_t)v) & 15))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: the state is NULL, or a pointer is not 16-byte aligned", fn);
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    const int grid = (int)std::min<int64_t>(cdiv(blocks, OC_THREADS / 32), (int64_t)pool->sm_count * 32);
    k_compact_export<<<grid, OC_THREADS, 0, (cudaStream_t)cuda_stream>>>((const uint8_t*)state, m, v, blocks);
    MARLAAS_LAUNCH_CHECK("k_compact_export");
    return MARLAAS_OK;
}

marlaas_status_t marlaas_adapter_pool_store(const marlaas_pool_t* pool, const void** At, const void** Bs) {
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "pool_store: pool is NULL");
    if (At) *At = pool->d_At;
    if (Bs) *Bs = pool->d_Bs;
    return MARLAAS_OK;
}

}  // extern "C"
