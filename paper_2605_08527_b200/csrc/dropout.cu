// The layer with dropout in its adapters, forward and backward.  With m the mask of token i (dropout.cuh), p_t the rate of its
// tenant and s'_t = s_t / (1 - p_t):
//     y_i = x_i W + s'_t ((m o x_i) A_t) B_t           dx_i = dy_i W^T + s'_t m o ((dy_i B_t^T) A_t^T)
//     dA_t = s'_t sum (m o x_i)^T (dy_i B_t^T)         dB_t = s'_t sum ((m o x_i) A_t)^T dy_i
// Dropping elements is exact and 1 / (1 - p_t) enters with the adapter's scale in fp32: the masked activations are never
// rounded anew.  The layer's own kernels run with s'_t in the place of s_t.
#include <string.h>

#include <algorithm>
#include <exception>
#include <vector>

#include "dropout.cuh"

namespace marlaas {

struct DropTables {
    uint32_t* limit;        // [cap]
    float* scale;           // [cap]  s'_t
    bf16* xd;               // [T][K] masked activations
    size_t total;
};
static DropTables carve_drop(const marlaas_pool* pool, int64_t T, char* base, size_t o) {
    DropTables t;
    auto take = [&](size_t bytes) { char* q = base ? base + o : nullptr; o += align_up(bytes, 256); return q; };
    t.limit = (uint32_t*)take(sizeof(uint32_t) * (size_t)pool->cap);
    t.scale = (float*)take(sizeof(float) * (size_t)pool->cap);
    t.xd = (bf16*)take(sizeof(bf16) * (size_t)(T > 0 ? T : 1) * (size_t)pool->K);
    t.total = o;
    return t;
}

// s'_t and the limits of all tenants.
__device__ __forceinline__ uint32_t drop_limit(float p) { return p > 0.f ? (uint32_t)rintf(fminf(p, 1.f) * 65536.f) : 0u; }
__global__ void k_drop_tables(int cap, const float* __restrict__ rates, const float* __restrict__ d_scale, uint32_t* __restrict__ limit,
                              float* __restrict__ scale) {
    const int t = blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= cap) return;
    const uint32_t l = drop_limit(rates[t]);
    limit[t] = l;
    scale[t] = l < 65536u ? d_scale[t] * (65536.f / (float)(65536u - l)) : 0.f;
}

// m o x, eight elements per thread and step.
__global__ void __launch_bounds__(256) k_drop_rows(int64_t T, int nvec, const bf16* __restrict__ x, int64_t ldx, const int32_t* __restrict__ tok_slot,
                                                   const uint32_t* __restrict__ limit, DropKey key, bf16* __restrict__ xd) {
    const int64_t n = T * nvec;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        const int64_t i = e / nvec;
        const int v = (int)(e - i * nvec);
        uint4 q = reinterpret_cast<const uint4*>(x + i * ldx)[v];
        const int t = tok_slot[i];
        const uint32_t l = t >= 0 ? limit[t] : 0u;
        if (l) q = drop_apply(q, drop_bits(key, (uint32_t)v, (uint32_t)i), l);
        reinterpret_cast<uint4*>(xd)[e] = q;
    }
}

static unsigned stream_grid(const marlaas_pool* pool, int64_t n) { return (unsigned)std::min<int64_t>(cdiv(n, 256), (int64_t)pool->sm_count * 16); }

static marlaas_status_t launch_drop_rows(const marlaas_pool* pool, int64_t T, const bf16* x, int64_t ldx, const Workspace& ws, const DropTables& d,
                                         const DropKey& key, cudaStream_t st) {
    const int nvec = (int)(pool->K / 8);
    k_drop_rows<<<stream_grid(pool, T * nvec), 256, 0, st>>>(T, nvec, x, ldx, ws.tok_slot, d.limit, key, d.xd);
    MARLAAS_LAUNCH_CHECK("k_drop_rows");
    return MARLAAS_OK;
}

static marlaas_status_t launch_drop_tables(const marlaas_pool* pool, const marlaas_dropout_t* drop, const DropTables& d, cudaStream_t st) {
    k_drop_tables<<<(unsigned)cdiv(pool->cap, 256), 256, 0, st>>>(pool->cap, drop->rates, pool->d_scale, d.limit, d.scale);
    MARLAAS_LAUNCH_CHECK("k_drop_tables");
    return MARLAAS_OK;
}

// h = (m o x) A of all projections.  From 512 tokens on the shrink kernels mask the rows themselves; for fewer, whose shrink reads a
// row once per rank, they are masked first.
static marlaas_status_t masked_shrink(const marlaas_pool* v, int64_t T, const bf16* x, int64_t ldx, const Workspace& ws, const DropTables& d,
                                      const DropKey& key, float* h, bool h_is_zero, bool rows_masked, cudaStream_t st) {
    marlaas_status_t rc;
    const int NP = v->P;
    const DropMask mask = {ws.tok_slot, d.limit, key};
    if (T < 512 && !rows_masked && (rc = launch_drop_rows(v, T, x, ldx, ws, d, key, st)) != MARLAAS_OK) return rc;
    if (NP > 1 && T >= 512 && shrink_split_sm100_parts_eligible(v, T, v->K, NP))
        return launch_shrink_split_sm100(v, T, x, ldx, v->K, v->d_At, v->K, ws, h, st, h_is_zero, NP, &mask);
    for (int p = 0; p < NP; ++p) {
        const bf16* At = v->d_At + (size_t)p * v->cap * v->RP * v->K;
        const Workspace wp = part_workspace(v, ws, p, T);
        float* hp = h + (size_t)p * T * v->RP;
        if (T < 512) rc = launch_shrink_hd(v, T, d.xd, v->K, v->K, At, v->K, wp, hp, st);
        else if (shrink_split_sm100_eligible(v, T, v->K)) rc = launch_shrink_split_sm100(v, T, x, ldx, v->K, At, v->K, wp, hp, st, h_is_zero, 1, &mask);
        else rc = launch_shrink_sm100(v, T, x, ldx, v->K, At, v->K, wp, hp, st, &mask);
        if (rc != MARLAAS_OK) return rc;
    }
    return MARLAAS_OK;
}

static bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

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
    marlaas_pool v;
    scaled_view(pool, d.scale, &v);
    float* h = h_save ? h_save : ws.h;
    const bool pre_zero = T >= 512 && shrink_split_sm100_eligible(pool, T, pool->K);       // (before the plan: see lora_forward)
    if (pre_zero) MARLAAS_CUDA_TRY(cudaMemsetAsync(h, 0, sizeof(float) * (size_t)pool->P * T * pool->RP, st));
    if ((rc = launch_drop_tables(pool, drop, d, st)) != MARLAAS_OK) return rc;
    if ((rc = make_plan(&v, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
    if ((rc = masked_shrink(&v, T, (const bf16*)x, ldx, ws, d, drop_key(drop), h, pre_zero, false, st)) != MARLAAS_OK) return rc;
    GemmOperands o;
    forward_operands(pool, T, (const bf16*)x, ldx, (const bf16*)W, ldw, (bf16*)y, ldy, ws, &o);
    rc = (pool->P > 1 || gemm2_sm100_eligible(pool, T)) ? launch_gemm2_sm100(&v, o, st) : launch_gemm_sm100(&v, o, st);
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
    const DropKey key = drop_key(drop);
    marlaas_pool v;
    scaled_view(pool, d.scale, &v);
    const int NP = pool->P;
    // One kernel after another on the caller's stream.
    const bool pre_zero = T >= 512 && NP == 1 && (dx || want_dA) && shrink_split_sm100_eligible(pool, T, pool->N);
    if (pre_zero) MARLAAS_CUDA_TRY(cudaMemsetAsync(ws.g, 0, sizeof(float) * (size_t)T * pool->RP, st));
    if ((rc = launch_drop_tables(pool, drop, d, st)) != MARLAAS_OK) return rc;
    if (T > 0) {
        if ((rc = make_plan(&v, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
        if (dx || want_dA)
            for (int p = 0; p < NP; ++p) {
                const int64_t c0 = pool->part_begin[p], Np = pool->part_begin[p + 1] - c0;
                const Workspace wp = part_workspace(pool, ws, p, T);
                if ((rc = shrink(&v, T, (const bf16*)dy + c0, lddy, Np, pool->d_Bs + c0, pool->ldB, wp, wp.g, st, pre_zero)) != MARLAAS_OK) return rc;
            }
        if (dx) {
            GemmOperands o;
            backward_operands(pool, T, (const bf16*)W, ldw, (const bf16*)dy, lddy, (bf16*)dx, lddx, ws, &o);
            if ((rc = launch_gemm2_dropped(&v, o, DropMask{ws.tok_slot, d.limit, key}, st)) != MARLAAS_OK) return rc;
        }
        if (want_dA && (rc = launch_drop_rows(pool, T, (const bf16*)x, ldx, ws, d, key, st)) != MARLAAS_OK) return rc;
        if (want_dB && !h_saved && (rc = masked_shrink(&v, T, (const bf16*)x, ldx, ws, d, key, ws.h, false, want_dA, st)) != MARLAAS_OK) return rc;
    }
    if ((want_dA || want_dB) &&
        (rc = adapter_gradients(&v, T, d.xd, pool->K, (const bf16*)dy, lddy, dA_slots, dB_slots, seg, h_saved ? h_saved : ws.h, ws, acc, st)) != MARLAAS_OK)
        return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "lora_backward_dropout: %s", e.what());
}

}  // extern "C"
