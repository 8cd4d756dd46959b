// The layer with dropout in its adapters, forward and backward.  With m the mask of token i (dropout.cuh), p_t the rate of its
// tenant and s'_t = s_t / (1 - p_t):
//     y_i = x_i W + s'_t ((m o x_i) A_t) B_t           dx_i = dy_i W^T + s'_t m o ((dy_i B_t^T) A_t^T)
//     dA_t = s'_t sum (m o x_i)^T (dy_i B_t^T)         dB_t = s'_t sum ((m o x_i) A_t)^T dy_i
// Dropping elements is exact and 1 / (1 - p_t) enters with the adapter's scale in fp32: the masked activations are never
// rounded anew.  The layer's own kernels run with s'_t in the place of s_t; no masked copy of x is written but for batches whose
// tenants mix too finely for the tensor-core reductions.
// The products bound it, as they do the layer: forward 8192 x 4096 x 4096 with 32 tenants of rank 16 250 us (the product 180 at full
// clocks, the masked shrink 40, of which the masks' random numbers are 8), backward 320 us (dx 186, its masks 8 of them; shrink 33;
// the reductions 35 and 42).  All kernels of a call follow one another on the caller's stream: the reductions beside the dx product
// on a second stream measured 4 % less, but once in some 12000 calls under a deep queue that form stopped making progress.
#include <string.h>

#include <algorithm>
#include <exception>
#include <vector>

#include "dropout.cuh"

namespace marlaas {

// Fewer tokens: kernels of a CTA per token and per slot, in as few launches as there are steps; a thread per token is what the
// gradients' kernel has.  Against the kernels for many tokens (captured, rank 16): 512 x 512 forward 64 tokens 13 us for 22, 511
// tokens 15 for 24; backward 29 for 39 and 52 for 47; 4096 x 4096 forward 46 for 52 and 51 for 55, backward 67 for 71 and 88 for 78.
constexpr int64_t DROP_SMALL_T = 512;

struct DropTables {
    float* scale;           // [cap]  s'_t
    bf16* xd;               // [T][K] masked activations
    size_t total;
};
static DropTables carve_drop(const marlaas_pool* pool, int64_t T, char* base, size_t o) {
    DropTables t;
    auto take = [&](size_t bytes) { char* q = base ? base + o : nullptr; o += align_up(bytes, 256); return q; };
    t.scale = (float*)take(sizeof(float) * (size_t)pool->cap);
    t.xd = (bf16*)take(sizeof(bf16) * (size_t)(T > 0 ? T : 1) * (size_t)pool->K);
    t.total = o;
    return t;
}

// What the kernels of a batch of many tokens need before them: s'_t, and zeros in the n16 16-byte words that the split shrink adds to.
__global__ void __launch_bounds__(256) k_drop_begin(int cap, const float* __restrict__ rates, const float* __restrict__ d_scale, float* __restrict__ scale,
                                                    uint4* __restrict__ zero, int64_t n16) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at < cap) scale[at] = drop_scale(d_scale[at], drop_limit(rates[at]));
    for (int64_t i = at; i < n16; i += (int64_t)gridDim.x * 256) zero[i] = make_uint4(0u, 0u, 0u, 0u);
}

// m o x, eight elements per thread and step.
__global__ void __launch_bounds__(256) k_drop_rows(int64_t T, int nvec, const bf16* __restrict__ x, int64_t ldx, const DropMask m, bf16* __restrict__ xd) {
    const int64_t n = T * nvec;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        const int64_t i = e / nvec;
        const int v = (int)(e - i * nvec);
        uint4 q = reinterpret_cast<const uint4*>(x + i * ldx)[v];
        const int t = m.tok_slot[i];
        const uint32_t l = t >= 0 ? drop_limit(m.rates[t]) : 0u;
        if (l) q = drop_apply(q, drop_bits(m.key, (uint32_t)v, (uint32_t)i), l);
        reinterpret_cast<uint4*>(xd)[e] = q;
    }
}

static marlaas_status_t launch_drop_rows(const marlaas_pool* pool, int64_t T, const bf16* x, int64_t ldx, const DropMask& m, bf16* xd, cudaStream_t st) {
    const int nvec = (int)(pool->K / 8);
    const unsigned grid = (unsigned)std::min<int64_t>(cdiv(T * nvec, 256), (int64_t)pool->sm_count * 16);
    k_drop_rows<<<grid, 256, 0, st>>>(T, nvec, x, ldx, m, xd);
    MARLAAS_LAUNCH_CHECK("k_drop_rows");
    return MARLAAS_OK;
}

// ---- few tokens ----
// h = (m o x) A_t (MASK) or g = dy B_t^T, a CTA per token: the row, masked, in shared memory, four ranks per warp at a time; with the
// token's row of the products' low-rank operand, bf16(s'_t h) in its tenant's unit columns and zeros in the tile's others.
template <bool MASK>
__global__ void __launch_bounds__(128) k_drop_shrink(int D, const bf16* __restrict__ src, int64_t ld, const bf16* __restrict__ store, int64_t sld,
                                                     const DropMask m, const int32_t* __restrict__ tok_uoff, const int32_t* __restrict__ tile_nunits,
                                                     const int32_t* __restrict__ d_rank, const float* __restrict__ d_scale, int RP, int cap, int hd_cols,
                                                     float* __restrict__ out, bf16* __restrict__ hd) {
    extern __shared__ uint4 s_row[];        // MASK: [D / 8]
    __shared__ float sh[128];
    const int64_t i = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nvec = D / 8;
    const int t = m.tok_slot[i], r = t >= 0 && t < cap ? d_rank[t] : 0;
    const uint32_t limit = r > 0 ? drop_limit(m.rates[t]) : 0u;
    const float s = r > 0 ? drop_scale(d_scale[t], limit) : 0.f;
    const uint4* row = reinterpret_cast<const uint4*>(src + i * ld);
    if (MASK && r > 0) {
        for (int v = tid; v < nvec; v += 128) s_row[v] = limit ? drop_apply(row[v], drop_bits(m.key, (uint32_t)v, (uint32_t)i), limit) : row[v];
        __syncthreads();
        row = s_row;
    }
    for (int j0 = warp * 4; j0 < RP; j0 += 16) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        if (j0 < r) {       // (rows of the store from a tenant's rank to its next multiple of 16 are zeros)
            const bf16* a = store + ((size_t)t * RP + j0) * sld;
            for (int v = lane; v < nvec; v += 32) {
                const uint4 q = row[v];
                const uint32_t* x = &q.x;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 b = *reinterpret_cast<const uint4*>(a + k * sld + v * 8);
                    const uint32_t* y = &b.x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[k] = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), acc[k]);
                        acc[k] = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), acc[k]);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            for (int o = 16; o > 0; o >>= 1) acc[k] += __shfl_xor_sync(0xffffffffu, acc[k], o);
            if (lane == 0) sh[j0 + k] = out[i * RP + j0 + k] = j0 + k < r ? acc[k] : 0.f;
        }
    }
    __syncthreads();
    const int nun = tile_nunits[i >> 8], uo = r > 0 ? tok_uoff[i] : -1;
    const int own0 = uo * 16, own1 = own0 + ((r + 15) >> 4) * 16;
    for (int c = tid * 8; c < nun * 16; c += 128 * 8) {
        uint4 o = make_uint4(0u, 0u, 0u, 0u);
        if (uo >= 0 && c >= own0 && c < own1) {
            uint32_t* w = &o.x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                __nv_bfloat162 p = __floats2bfloat162_rn(s * sh[c - own0 + 2 * e], s * sh[c - own0 + 2 * e + 1]);
                w[e] = *reinterpret_cast<uint32_t*>(&p);
            }
        }
        *reinterpret_cast<uint4*>(hd + i * hd_cols + c) = o;
    }
}

// dB and dA of one tenant, 256 columns and 16 ranks per CTA: it lists the tenant's tokens and adds up their products in fp32, a
// thread eight columns of four ranks; DROP_PARTS parts of the CTA take the tokens in turn, and their sums are added in order.
// Bound by the latency of a token's row: four rows of each part are on their way at a time (300 x 2048 x 2048, rank 32, 16 tenants:
// 37 us; with one part per CTA 75).  The first CTAs along x do dB
// (columns of dy), the others dA (of x, masked).
constexpr int DROP_PARTS = 4;
constexpr int DROP_INLINE_SLOTS = 64;
struct DropGrads {
    int T, cap, RP, K, N, tiles_b;
    const bf16* x; int64_t ldx;
    const bf16* dy; int64_t lddy;
    const float* g;
    const float* h;
    DropMask m;
    const int32_t* d_rank;
    const float* d_scale;
    float* const* dA_ptrs;      // device tables, or NULL: those below
    float* const* dB_ptrs;
    int accumulate;
    float* dA[DROP_INLINE_SLOTS];
    float* dB[DROP_INLINE_SLOTS];
};
__global__ void __launch_bounds__(128 * DROP_PARTS) k_drop_grads(const __grid_constant__ DropGrads a) {
    constexpr int WARPS = 4 * DROP_PARTS;
    __shared__ int s_tok[DROP_SMALL_T], s_warp[WARPS];
    __shared__ float s_acc[32][128];
    const int t = blockIdx.y, j0 = blockIdx.z * 16, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool is_b = (int)blockIdx.x < a.tiles_b;
    float* out = is_b ? (a.dB_ptrs ? a.dB_ptrs[t] : a.dB[t]) : (a.dA_ptrs ? a.dA_ptrs[t] : a.dA[t]);
    const int r = a.d_rank[t];
    if (!out || j0 >= r) return;
    static_assert(128 * DROP_PARTS == DROP_SMALL_T, "a thread per token");
    const bool mine = tid < a.T && a.m.tok_slot[tid] == t;
    const unsigned bal = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) s_warp[warp] = __popc(bal);
    __syncthreads();
    int n = 0, at = __popc(bal & ((1u << lane) - 1u));
    for (int w = 0; w < WARPS; ++w) {
        at += w < warp ? s_warp[w] : 0;
        n += s_warp[w];
    }
    if (mine) s_tok[at] = tid;
    __syncthreads();
    const int C = is_b ? a.N : a.K, c = ((int)blockIdx.x - (is_b ? 0 : a.tiles_b)) * 256 + lane * 8, part = warp >> 2, j = j0 + (warp & 3) * 4;
    const bool on = c < C && j < r;
    const uint32_t limit = drop_limit(a.m.rates[t]);
    const float s = drop_scale(a.d_scale[t], limit);
    const bf16* src = (is_b ? a.dy : a.x) + c;
    const int64_t ld = is_b ? a.lddy : a.ldx;
    const float* v = (is_b ? a.h : a.g) + j;
    const bool masked = !is_b && limit > 0;
    float acc[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[k][e] = 0.f;
    constexpr int U = 4;
    if (on) {
        for (int q0 = part; q0 < n; q0 += DROP_PARTS * U) {
            uint4 x[U];
            float4 f[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int q = q0 + u * DROP_PARTS;
                if (q < n) {
                    const int i = s_tok[q];
                    x[u] = *reinterpret_cast<const uint4*>(src + i * ld);
                    f[u] = *reinterpret_cast<const float4*>(v + (int64_t)i * a.RP);
                } else {
                    x[u] = make_uint4(0u, 0u, 0u, 0u);
                    f[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int q = q0 + u * DROP_PARTS;
                if (masked && q < n) x[u] = drop_apply(x[u], drop_bits(a.m.key, (uint32_t)(c / 8), (uint32_t)s_tok[q]), limit);
                const uint32_t* w = &x[u].x;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
                    acc[0][e] = fmaf(f[u].x, z, acc[0][e]);
                    acc[1][e] = fmaf(f[u].y, z, acc[1][e]);
                    acc[2][e] = fmaf(f[u].z, z, acc[2][e]);
                    acc[3][e] = fmaf(f[u].w, z, acc[3][e]);
                }
            }
        }
    }
    for (int p = 0; p < DROP_PARTS; ++p) {      // the parts' sums in their order
        if (part == p) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float* to = &s_acc[k * 8 + e][tid & 127];
                    *to = p == 0 ? acc[k][e] : *to + acc[k][e];
                }
        }
        __syncthreads();
    }
    if (!on || (n == 0 && a.accumulate)) return;
    // part k writes rank j + k: eight columns of dB's row, or one rank of eight of dA's
    if (j + part >= r) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float* to = is_b ? out + (size_t)(j + part) * C + c + e : out + (size_t)(c + e) * r + j + part;
        const float z = s * s_acc[part * 8 + e][tid & 127];
        *to = a.accumulate ? *to + z : z;
    }
}

// h = (m o x) A of all projections (x given), or g = dy B^T (dy given), and the low-rank operand.
static marlaas_status_t small_shrink(const marlaas_pool* pool, int64_t T, const bf16* x, int64_t ldx, const bf16* dy, int64_t lddy, const Workspace& ws,
                                     const DropTables& d, const DropMask& m, float* out, cudaStream_t st) {
    // a row of more than 96 K elements does not fit shared memory: masked in the workspace first
    const bool wide = x && pool->K > 96 * 1024;
    marlaas_status_t rc;
    if (wide) {
        if ((rc = launch_drop_rows(pool, T, x, ldx, m, d.xd, st)) != MARLAAS_OK) return rc;
        x = d.xd;
        ldx = pool->K;
    }
    for (int p = 0; p < pool->P; ++p) {
        const int64_t c0 = pool->part_begin[p];
        const Workspace wp = part_workspace(pool, ws, p, T);
        const int D = (int)(x ? pool->K : pool->part_begin[p + 1] - c0);
        const bf16 *src = x ? x : dy + c0, *store = x ? pool->d_At + (size_t)p * pool->cap * pool->RP * pool->K : pool->d_Bs + c0;
        const int64_t ld = x ? ldx : lddy, sld = x ? pool->K : pool->ldB;
        float* o = out + (size_t)p * T * pool->RP;
        if (x && !wide) {
            static bool attr_set[64] = {};
            if (pool->device >= 64 || !attr_set[pool->device]) {
                MARLAAS_CUDA_TRY(cudaFuncSetAttribute(k_drop_shrink<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * 96 * 1024));
                if (pool->device < 64) attr_set[pool->device] = true;
            }
            k_drop_shrink<true><<<(unsigned)T, 128, (size_t)D * 2, st>>>(D, src, ld, store, sld, m, wp.tok_uoff, wp.tile_nunits, pool->d_rank, pool->d_scale,
                                                                         pool->RP, pool->cap, ws.umax * 16, o, wp.hd);
        } else {
            k_drop_shrink<false><<<(unsigned)T, 128, 0, st>>>(D, src, ld, store, sld, m, wp.tok_uoff, wp.tile_nunits, pool->d_rank, pool->d_scale,
                                                              pool->RP, pool->cap, ws.umax * 16, o, wp.hd);
        }
        MARLAAS_LAUNCH_CHECK("k_drop_shrink");
    }
    return MARLAAS_OK;
}

static marlaas_status_t small_gradients(const marlaas_pool* pool, int64_t T, const bf16* x, int64_t ldx, const bf16* dy, int64_t lddy,
                                        float* const* dA_slots, float* const* dB_slots, const float* h, const Workspace& ws, const DropMask& m,
                                        bool accumulate, cudaStream_t st) {
    const size_t plane = (size_t)T * pool->RP;
    std::vector<float*> tA((size_t)pool->cap, nullptr), tB((size_t)pool->cap, nullptr);
    for (int p = 0; p < pool->P; ++p) {
        const int64_t c0 = pool->part_begin[p], Np = pool->part_begin[p + 1] - c0;
        for (int s = 0; s < pool->cap; ++s) {       // block p of dA_t is [K][r_t], block p of dB_t is [r_t][N_p]
            const size_t r = (size_t)pool->slots[s].rank;
            tA[s] = dA_slots && dA_slots[s] ? dA_slots[s] + (size_t)p * pool->K * r : nullptr;
            tB[s] = dB_slots && dB_slots[s] ? dB_slots[s] + r * (size_t)c0 : nullptr;
        }
        DropGrads a;
        memset(&a, 0, sizeof(a));
        a.T = (int)T; a.cap = pool->cap; a.RP = pool->RP; a.K = (int)pool->K; a.N = (int)Np;
        a.tiles_b = dB_slots ? (int)cdiv(Np, 256) : 0;
        const int tiles_a = dA_slots ? (int)cdiv(pool->K, 256) : 0;
        a.x = x; a.ldx = ldx; a.dy = dy + c0; a.lddy = lddy; a.g = ws.g + p * plane; a.h = h ? h + p * plane : nullptr; a.m = m;
        a.d_rank = pool->d_rank; a.d_scale = pool->d_scale; a.accumulate = accumulate ? 1 : 0;
        if (pool->cap <= DROP_INLINE_SLOTS) {
            std::copy(tA.begin(), tA.end(), a.dA);
            std::copy(tB.begin(), tB.end(), a.dB);
        } else {
            MARLAAS_CUDA_TRY(cudaMemcpyAsync(ws.dA_ptrs, tA.data(), sizeof(float*) * (size_t)pool->cap, cudaMemcpyHostToDevice, st));
            MARLAAS_CUDA_TRY(cudaMemcpyAsync(ws.dB_ptrs, tB.data(), sizeof(float*) * (size_t)pool->cap, cudaMemcpyHostToDevice, st));
            a.dA_ptrs = ws.dA_ptrs;
            a.dB_ptrs = ws.dB_ptrs;
        }
        k_drop_grads<<<dim3((unsigned)(a.tiles_b + tiles_a), (unsigned)pool->cap, (unsigned)(pool->RP / 16)), 128 * DROP_PARTS, 0, st>>>(a);
        MARLAAS_LAUNCH_CHECK("k_drop_grads");
    }
    return MARLAAS_OK;
}

// ---- many tokens ----
// h = (m o x) A of all projections by the shrink kernels, which mask the rows themselves.
static marlaas_status_t masked_shrink(const marlaas_pool* v, int64_t T, const bf16* x, int64_t ldx, const Workspace& ws, const DropMask& m, float* h,
                                      bool h_is_zero, cudaStream_t st) {
    const int NP = v->P;
    if (NP > 1 && shrink_split_sm100_parts_eligible(v, T, v->K, NP))
        return launch_shrink_split_sm100(v, T, x, ldx, v->K, v->d_At, v->K, ws, h, st, h_is_zero, NP, &m);
    for (int p = 0; p < NP; ++p) {
        const bf16* At = v->d_At + (size_t)p * v->cap * v->RP * v->K;
        const Workspace wp = part_workspace(v, ws, p, T);
        float* hp = h + (size_t)p * T * v->RP;
        const marlaas_status_t rc = shrink_split_sm100_eligible(v, T, v->K, true)
                                        ? launch_shrink_split_sm100(v, T, x, ldx, v->K, At, v->K, wp, hp, st, h_is_zero, 1, &m)
                                        : launch_shrink_sm100(v, T, x, ldx, v->K, At, v->K, wp, hp, st, h_is_zero, &m);
        if (rc != MARLAAS_OK) return rc;
    }
    return MARLAAS_OK;
}

// zero: rank vectors of n floats (a multiple of 16) to clear, or NULL
static marlaas_status_t launch_drop_begin(const marlaas_pool* pool, const marlaas_dropout_t* drop, const DropTables& d, float* zero, size_t n,
                                          cudaStream_t st) {
    const int64_t n16 = zero ? (int64_t)(n / 4) : 0;
    const unsigned grid = (unsigned)std::max<int64_t>(cdiv(pool->cap, 256), std::min<int64_t>(cdiv(n16, 256), (int64_t)pool->sm_count * 8));
    k_drop_begin<<<grid, 256, 0, st>>>(pool->cap, drop->rates, pool->d_scale, d.scale, (uint4*)zero, n16);
    MARLAAS_LAUNCH_CHECK("k_drop_begin");
    return MARLAAS_OK;
}

static marlaas_status_t check_drop(const char* fn, const marlaas_pool* pool, int64_t T, const marlaas_dropout_t* drop, uint32_t flags, uint32_t allowed,
                                   void* workspace, size_t workspace_bytes) {
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (T < 0 || T >= (1ll << 31)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: T out of range", fn);
    if (flags & ~allowed) return fail(MARLAAS_ERR_INVALID_ARG, "%s: a flag does not apply to this call", fn);
    if (!drop || !drop->rates || misaligned(drop->rates, 4)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: the dropout rates are NULL or misaligned", fn);
    if (!workspace || misaligned(workspace, 256)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: workspace NULL or misaligned", fn);
    const size_t need = marlaas_lora_dropout_workspace_bytes(pool, T);
    if (workspace_bytes < need)
        return fail(MARLAAS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < required %zu", fn, workspace_bytes, need);
    return MARLAAS_OK;
}

static DropKey drop_key(const marlaas_dropout_t* d) {
    return DropKey{(uint32_t)d->seed, (uint32_t)(d->seed >> 32), (uint32_t)d->offset, (uint32_t)(d->offset >> 32)};
}

}  // namespace marlaas

using namespace marlaas;

extern "C" {

size_t marlaas_lora_dropout_workspace_bytes(const marlaas_pool_t* pool, int64_t T) {
    if (!pool || T < 0 || T >= (1ll << 31)) return 0;
    return carve_drop(pool, T, nullptr, carve_workspace(pool, T, nullptr).total).total;
}

marlaas_status_t marlaas_lora_forward_dropout(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx, const void* W, int64_t ldw, void* y,
                                              int64_t ldy, const marlaas_segments_t* seg, const marlaas_dropout_t* drop, float* h_save,
                                              void* workspace, size_t workspace_bytes, uint32_t flags, void* cuda_stream) try {
    const char* fn = "lora_forward_dropout";
    marlaas_status_t rc = check_drop(fn, pool, T, drop, flags, MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC, workspace, workspace_bytes);
    if (rc != MARLAAS_OK) return rc;
    if (T == 0) return MARLAAS_OK;
    if ((rc = check_matrix(fn, "x", x, ldx, pool->K)) != MARLAAS_OK) return rc;
    if ((rc = check_matrix(fn, "W", W, ldw, pool->N)) != MARLAAS_OK) return rc;
    if ((rc = check_matrix(fn, "y", y, ldy, pool->N)) != MARLAAS_OK) return rc;
    if (misaligned(h_save, 16)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: h_save is not 16-byte aligned", fn);
    std::vector<int32_t> host_ts;
    if ((rc = check_segments(fn, pool, T, seg, flags, &host_ts)) != MARLAAS_OK) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    const Workspace ws = carve_workspace(pool, T, workspace);
    const DropTables d = carve_drop(pool, T, (char*)workspace, ws.total);
    const DropMask mask = {ws.tok_slot, drop->rates, drop_key(drop)};
    float* h = h_save ? h_save : ws.h;
    if (T < DROP_SMALL_T) {
        if ((rc = make_plan(pool, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
        if ((rc = small_shrink(pool, T, (const bf16*)x, ldx, nullptr, 0, ws, d, mask, h, st)) != MARLAAS_OK) return rc;
    } else {
        marlaas_pool v;
        scaled_view(pool, d.scale, &v);
        if ((rc = launch_drop_begin(pool, drop, d, h, (size_t)pool->P * T * pool->RP, st)) != MARLAAS_OK) return rc;
        if ((rc = make_plan(pool, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
        if ((rc = masked_shrink(&v, T, (const bf16*)x, ldx, ws, mask, h, true, st)) != MARLAAS_OK) return rc;
    }
    GemmOperands o;
    forward_operands(pool, T, (const bf16*)x, ldx, (const bf16*)W, ldw, (bf16*)y, ldy, ws, &o);
    rc = (pool->P > 1 || gemm2_sm100_eligible(pool, T)) ? launch_gemm2_sm100(pool, o, st) : launch_gemm_sm100(pool, o, st);
    if (rc != MARLAAS_OK) return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "lora_forward_dropout: %s", e.what());
}

marlaas_status_t marlaas_lora_backward_dropout(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx, const void* W, int64_t ldw,
                                               const void* dy, int64_t lddy, void* dx, int64_t lddx, float* const* dA_slots,
                                               float* const* dB_slots, const marlaas_segments_t* seg, const marlaas_dropout_t* drop,
                                               const float* h_saved, void* workspace, size_t workspace_bytes, uint32_t flags,
                                               void* cuda_stream) try {
    const char* fn = "lora_backward_dropout";
    marlaas_status_t rc = check_drop(fn, pool, T, drop, flags, MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC | MARLAAS_FLAG_ACCUMULATE, workspace,
                                     workspace_bytes);
    if (rc != MARLAAS_OK) return rc;
    const bool want_dA = dA_slots != nullptr, want_dB = dB_slots != nullptr, acc = (flags & MARLAAS_FLAG_ACCUMULATE) != 0;
    if (T > 0) {
        if ((rc = check_matrix(fn, "W", W, ldw, pool->N)) != MARLAAS_OK) return rc;
        if ((rc = check_matrix(fn, "dy", dy, lddy, pool->N)) != MARLAAS_OK) return rc;
        if (dx && (rc = check_matrix(fn, "dx", dx, lddx, pool->K)) != MARLAAS_OK) return rc;
        if ((want_dA || (want_dB && !h_saved)) && (rc = check_matrix(fn, "x", x, ldx, pool->K)) != MARLAAS_OK) return rc;
    }
    if (misaligned(h_saved, 16)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: h_saved is not 16-byte aligned", fn);
    for (int s = 0; s < pool->cap; ++s)
        if ((want_dA && misaligned(dA_slots[s], 4)) || (want_dB && misaligned(dB_slots[s], 4)))
            return fail(MARLAAS_ERR_INVALID_ARG, "%s: a gradient of slot %d is misaligned", fn, s);
    std::vector<int32_t> host_ts;
    if ((rc = check_segments(fn, pool, T, seg, flags, &host_ts)) != MARLAAS_OK) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    if ((want_dA || want_dB) && (rc = reject_captured_tables(fn, pool, st)) != MARLAAS_OK) return rc;
    const Workspace ws = carve_workspace(pool, T, workspace);
    const DropTables d = carve_drop(pool, T, (char*)workspace, ws.total);
    const DropMask mask = {ws.tok_slot, drop->rates, drop_key(drop)};
    const int NP = pool->P;
    const float* h = h_saved ? h_saved : ws.h;
    auto product = [&]() -> marlaas_status_t {
        if (!dx) return MARLAAS_OK;
        GemmOperands o;
        backward_operands(pool, T, (const bf16*)W, ldw, (const bf16*)dy, lddy, (bf16*)dx, lddx, ws, &o);
        return launch_gemm2_dropped(pool, o, mask, st);
    };
    // one kernel after another on the caller's stream
    if (T < DROP_SMALL_T) {
        if (T > 0) {
            if ((rc = make_plan(pool, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
            if ((dx || want_dA) && (rc = small_shrink(pool, T, nullptr, 0, (const bf16*)dy, lddy, ws, d, mask, ws.g, st)) != MARLAAS_OK) return rc;
            if ((rc = product()) != MARLAAS_OK) return rc;
            if (want_dB && !h_saved && (rc = small_shrink(pool, T, (const bf16*)x, ldx, nullptr, 0, ws, d, mask, ws.h, st)) != MARLAAS_OK) return rc;
        }
        if ((want_dA || want_dB) && (rc = small_gradients(pool, T, (const bf16*)x, ldx, (const bf16*)dy, lddy, dA_slots, dB_slots, h, ws, mask, acc, st)) != MARLAAS_OK)
            return rc;
        return finish(pool, flags, st);
    }
    marlaas_pool v;
    scaled_view(pool, d.scale, &v);
    if ((rc = launch_drop_begin(pool, drop, d, dx || want_dA ? ws.g : nullptr, (size_t)NP * T * pool->RP, st)) != MARLAAS_OK) return rc;
    if ((rc = make_plan(pool, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
    if (dx || want_dA)
        for (int p = 0; p < NP; ++p) {
            const int64_t c0 = pool->part_begin[p], Np = pool->part_begin[p + 1] - c0;
            const Workspace wp = part_workspace(pool, ws, p, T);
            rc = shrink_split_sm100_eligible(pool, T, Np, true)
                     ? launch_shrink_split_sm100(&v, T, (const bf16*)dy + c0, lddy, Np, pool->d_Bs + c0, pool->ldB, wp, wp.g, st, true)
                     : launch_shrink_sm100(&v, T, (const bf16*)dy + c0, lddy, Np, pool->d_Bs + c0, pool->ldB, wp, wp.g, st, true);
            if (rc != MARLAAS_OK) return rc;
        }
    if ((rc = product()) != MARLAAS_OK) return rc;
    // the reduction for dA masks the rows itself, but for batches whose tenants may mix too finely for it
    const bool fits = adapter_gradients_fit(pool, T, seg, ws);
    if (want_dA && !fits && (rc = launch_drop_rows(pool, T, (const bf16*)x, ldx, mask, d.xd, st)) != MARLAAS_OK) return rc;
    if (want_dB && !h_saved && (rc = masked_shrink(&v, T, (const bf16*)x, ldx, ws, mask, ws.h, false, st)) != MARLAAS_OK) return rc;
    const DropMask masked = {mask.tok_slot, nullptr, mask.key};
    if ((want_dA || want_dB) &&
        (rc = adapter_gradients(&v, T, fits ? (const bf16*)x : d.xd, fits ? ldx : pool->K, (const bf16*)dy, lddy, dA_slots, dB_slots, seg, h, ws, acc,
                                st, fits ? &mask : &masked)) != MARLAAS_OK)
        return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "lora_backward_dropout: %s", e.what());
}

}  // extern "C"
