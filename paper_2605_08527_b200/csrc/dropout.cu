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

__global__ void k_drop_tables(int cap, const float* __restrict__ rates, const float* __restrict__ d_scale, uint32_t* __restrict__ limit,
                              float* __restrict__ scale) {
    const int t = blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= cap) return;
    const float p = rates[t];
    const uint32_t l = p > 0.f ? (uint32_t)rintf(fminf(p, 1.f) * 65536.f) : 0u;
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
    const int NP = pool->P;
    if ((rc = launch_drop_tables(pool, drop, d, st)) != MARLAAS_OK) return rc;
    if ((rc = make_plan(&v, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
    if ((rc = launch_drop_rows(pool, T, (const bf16*)x, ldx, ws, d, drop_key(drop), st)) != MARLAAS_OK) return rc;
    for (int p = 0; p < NP; ++p)
        if ((rc = shrink(&v, T, d.xd, pool->K, pool->K, pool->d_At + (size_t)p * pool->cap * pool->RP * pool->K, pool->K,
                         part_workspace(pool, ws, p, T), h + (size_t)p * T * pool->RP, st)) != MARLAAS_OK) return rc;
    GemmOperands o;
    forward_operands(pool, T, (const bf16*)x, ldx, (const bf16*)W, ldw, (bf16*)y, ldy, ws, &o);
    rc = (NP > 1 || gemm2_sm100_eligible(pool, T)) ? launch_gemm2_sm100(&v, o, st) : launch_gemm_sm100(&v, o, st);
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
    const size_t plane = (size_t)T * pool->RP;
    if ((rc = launch_drop_tables(pool, drop, d, st)) != MARLAAS_OK) return rc;
    if (T > 0 && (rc = make_plan(&v, T, seg, flags, host_ts, ws, st)) != MARLAAS_OK) return rc;
    auto masked_rows = [&](cudaStream_t s) { return launch_drop_rows(pool, T, (const bf16*)x, ldx, ws, d, key, s); };
    auto g_of_dy = [&]() -> marlaas_status_t {
        for (int p = 0; p < NP; ++p) {
            const int64_t c0 = pool->part_begin[p], Np = pool->part_begin[p + 1] - c0;
            const Workspace wp = part_workspace(pool, ws, p, T);
            const marlaas_status_t r = shrink(&v, T, (const bf16*)dy + c0, lddy, Np, pool->d_Bs + c0, pool->ldB, wp, wp.g, st);
            if (r != MARLAAS_OK) return r;
        }
        return MARLAAS_OK;
    };
    auto product = [&]() {
        GemmOperands o;
        backward_operands(pool, T, (const bf16*)W, ldw, (const bf16*)dy, lddy, (bf16*)dx, lddx, ws, &o);
        return launch_gemm2_dropped(&v, o, DropMask{ws.tok_slot, d.limit, key}, st);
    };
    // As in marlaas_lora_backward: where the reductions are certain to fit, all that the adapters' gradients need besides g is made
    // on the pool's side stream beside the dx product, and the reductions take the SMs that the product leaves (8192 x 4096 x 4096,
    // 32 tenants of rank 16: 364 us one after another, 321 so).
    const bool fits = grad_sm100_eligible(pool, T) && cdiv(T, 64) + (int64_t)seg->num_segments <= (int64_t)ws.max_copies;
    if (T >= 1024 && NP == 1 && fits && dx && (want_dA || want_dB) && (!want_dB || h_saved) && pool->cap <= 64) {
        if ((rc = make_side_stream(pool)) != MARLAAS_OK) return rc;
        cudaStream_t gs = pool->side;
        MARLAAS_CUDA_TRY(cudaEventRecord(pool->ev_fork, st));
        MARLAAS_CUDA_TRY(cudaStreamWaitEvent(gs, pool->ev_fork, 0));
        // whatever happens from here on, the side stream is joined again before the call returns
        auto work = [&]() -> marlaas_status_t {
            marlaas_status_t r;
            if ((r = launch_grad_plan(&v, T, ws, gs)) != MARLAAS_OK) return r;
            if (want_dB && (r = launch_grad_sm100(&v, T, pool->N, (const bf16*)dy, lddy, h_saved, nullptr, dB_slots, false, acc, ws, gs, ws.hm,
                                                  GRAD_PHASE_COPIES)) != MARLAAS_OK) return r;
            if ((r = g_of_dy()) != MARLAAS_OK) return r;
            MARLAAS_CUDA_TRY(cudaEventRecord(pool->ev_fork, st));
            if ((r = product()) != MARLAAS_OK) return r;
            if (want_dA && (r = masked_rows(gs)) != MARLAAS_OK) return r;
            MARLAAS_CUDA_TRY(cudaStreamWaitEvent(gs, pool->ev_fork, 0));
            if (want_dA && (r = launch_grad_sm100(&v, T, pool->K, d.xd, pool->K, ws.g, nullptr, dA_slots, true, acc, ws, gs, ws.hm2,
                                                  GRAD_PHASE_COPIES)) != MARLAAS_OK) return r;
            if (want_dB && (r = launch_grad_sm100(&v, T, pool->N, (const bf16*)dy, lddy, h_saved, nullptr, dB_slots, false, acc, ws, gs, ws.hm,
                                                  GRAD_PHASE_REDUCE)) != MARLAAS_OK) return r;
            if (want_dA && (r = launch_grad_sm100(&v, T, pool->K, d.xd, pool->K, ws.g, nullptr, dA_slots, true, acc, ws, gs, ws.hm2,
                                                  GRAD_PHASE_REDUCE | (want_dB ? GRAD_PHASE_EARLY : 0))) != MARLAAS_OK) return r;
            return MARLAAS_OK;
        };
        rc = work();
        MARLAAS_CUDA_TRY(cudaEventRecord(pool->ev_join, gs));
        MARLAAS_CUDA_TRY(cudaStreamWaitEvent(st, pool->ev_join, 0));
        if (rc != MARLAAS_OK) return rc;
        return finish(pool, flags, st);
    }
    if (T > 0) {
        if ((want_dA || (want_dB && !h_saved)) && (rc = masked_rows(st)) != MARLAAS_OK) return rc;
        if ((dx || want_dA) && (rc = g_of_dy()) != MARLAAS_OK) return rc;
        if (dx && (rc = product()) != MARLAAS_OK) return rc;
        if (want_dB && !h_saved)
            for (int p = 0; p < NP; ++p)
                if ((rc = shrink(&v, T, d.xd, pool->K, pool->K, pool->d_At + (size_t)p * pool->cap * pool->RP * pool->K, pool->K,
                                 part_workspace(pool, ws, p, T), ws.h + p * plane, st)) != MARLAAS_OK) return rc;
    }
    if ((want_dA || want_dB) &&
        (rc = adapter_gradients(&v, T, d.xd, pool->K, (const bf16*)dy, lddy, dA_slots, dB_slots, seg, h_saved ? h_saved : ws.h, ws, acc, st)) != MARLAAS_OK)
        return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "lora_backward_dropout: %s", e.what());
}

}  // extern "C"
