// The vocabulary head's logits for a few tokens (head.cu, up to HEAD_FEW_T of them): each tile of tensor memory holds 128 columns
// of the vocabulary by the tokens, W on the M side (MN-major, as it lies in memory) and the tokens on the N side, so that the tensor
// cores do 128 x np x 64 where a tile of 256 tokens by 256 columns would multiply mostly padding.  W's bytes bound it: the call for
// one token of 4096 x 131072 takes 198 us (164 of them the bytes, with the wide tiles 229), 32 x 1024 x 32768 27 us (10; 33), where
// two rounds of tiles on 148 SMs leave a quarter of the second empty.
//
// One CTA per SM takes tiles in turn: a TMA warp (the first tiles' W is on its way before the kernel that gathers the tokens has
// ended), an MMA thread, and four warps that read a tile from tensor memory (a thread a column), turn it over in shared memory and
// reduce it (a thread part of a token's columns).  A tile leaves as in the wide form: per token the largest logit as reference, the sum
// of the exponentials relative to it but for the target's, the target's logit, and for a gradient the exponentials in bf16.
#include <string.h>

#include "sm100_cluster.cuh"
#include "sm100_ptx.cuh"

namespace marlaas {
namespace sm100 {

constexpr int HF_THREADS = 192;
constexpr int HF_STAGES = 7;
constexpr int HF_COLS = 128;                                                // columns of the vocabulary per tile
constexpr uint32_t HF_A_BYTES = 2 * CHUNK_BYTES, HF_STAGE = HF_A_BYTES + HEAD_FEW_T * 128;
constexpr size_t HF_TILE_FLOATS = (size_t)HF_COLS * (HEAD_FEW_T + 1);
constexpr size_t HF_SMEM = 1024 + (size_t)HF_STAGES * HF_STAGE + HF_TILE_FLOATS * 4 + 256;
static_assert(HF_SMEM <= 227 * 1024, "shared memory of an SM");

struct HeadFewArgs {
    int T, V, np, nkb, tiles;
    bf16* E; int64_t lde;
    HeadEpilogue h;
    int32_t* status;
};

__device__ __forceinline__ void hf_ld_32x16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void hf_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }     // the four warps of the epilogue

__global__ void __launch_bounds__(HF_THREADS, 1)
k_head_few(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const HeadFewArgs g) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t s0 = smem_u32(smem);
    float* const s_tile = reinterpret_cast<float*>(smem + HF_STAGES * HF_STAGE);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + HF_STAGES * HF_STAGE + HF_TILE_FLOATS * 4);
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * HF_STAGES, bar_tfull = bar_empty + 8 * HF_STAGES, bar_tempty = bar_tfull + 16,
                   bar_drain = bar_tempty + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * HF_STAGES + 5);
    volatile int* abort_word = reinterpret_cast<volatile int*>(tmem_slot + 1);
    __shared__ float s_max[128], s_sum[128];
    __shared__ volatile int s_bad;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr uint32_t TMEM_COLS = 128;         // two buffers of 64 columns

    if (threadIdx.x == 0) {
        for (int s = 0; s < HF_STAGES; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_tfull + 8 * b, 1);
            mbar_init(bar_tempty + 8 * b, 4);
        }
        mbar_init(bar_drain, 1);
        *abort_word = 0;
        s_bad = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        prefetch_tmap(&tmW);
        prefetch_tmap(&tmX);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int mine = (int)blockIdx.x < g.tiles ? (g.tiles - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;     // tiles of this CTA
    const int steps = mine * g.nkb;
    const uint32_t x_bytes = (uint32_t)g.np * 128;

    if (warp == 0) {
        if (lane == 0) {    // ---- TMA producer
            auto load_w = [&](int it) {
                const int c0 = ((int)blockIdx.x + it / g.nkb * (int)gridDim.x) * HF_COLS, kb = it % g.nkb, s = it % HF_STAGES;
                const int chunks = min(2, (g.V - c0 + 63) / 64);
                const uint32_t full = bar_full + 8 * s;
                mbar_expect_tx(full, (uint32_t)chunks * CHUNK_BYTES + x_bytes);
                for (int c = 0; c < chunks; ++c) tma_load_2d(s0 + s * HF_STAGE + c * CHUNK_BYTES, &tmW, full, c0 + c * 64, kb * 64);
            };
            auto load_x = [&](int it) {
                const int s = it % HF_STAGES;
                tma_load_2d(s0 + s * HF_STAGE + HF_A_BYTES, &tmX, bar_full + 8 * s, it % g.nkb * 64, 0);
            };
            const int early = min(steps, HF_STAGES);
            for (int it = 0; it < early; ++it) load_w(it);
            dk_wait_prerequisites();
            dk_launch_dependents();
            for (int it = 0; it < early; ++it) load_x(it);
            int it = early;
            bool ok = true;
            for (; it < steps; ++it) {
                if (!(ok = mbar_wait(bar_empty + 8 * (it % HF_STAGES), (uint32_t)(it / HF_STAGES - 1) & 1u, abort_word, 71))) break;
                load_w(it);
                load_x(it);
            }
            if (!ok) {      // the copies in flight land before the CTA ends
                for (int j = max(0, it - HF_STAGES); j < it; ++j) {
                    const unsigned long long t0 = global_ns();
                    while (!mbar_try_wait(bar_full + 8 * (j % HF_STAGES), (uint32_t)(j / HF_STAGES) & 1u) && global_ns() - t0 < WAIT_LIMIT_NS) {
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {    // ---- MMA: M = 128 columns of W (MN-major), N = np tokens (K-major)
            const uint32_t idesc = make_idesc(g.np, 0) | (1u << 15);
            bool ok = true;
            int it = 0;
            for (int j = 0; j < mine && ok; ++j) {
                const uint32_t b = j & 1;
                if (!(ok = mbar_wait(bar_tempty + 8 * b, ((uint32_t)(j >> 1) & 1u) ^ 1u, abort_word, 72))) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + b * 64;
                uint32_t acc = 0;
                for (int kb = 0; kb < g.nkb; ++kb, ++it) {
                    const int s = it % HF_STAGES;
                    if (!(ok = mbar_wait(bar_full + 8 * s, (uint32_t)(it / HF_STAGES) & 1u, abort_word, 73))) break;
                    tc_fence_after();
                    const uint64_t da = desc_mn_major(s0 + s * HF_STAGE, CHUNK_BYTES), db = desc_k_major(s0 + s * HF_STAGE + HF_A_BYTES);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        tc_mma_bf16(d_tmem, da + (uint64_t)(u * (UNIT_BYTES >> 4)), db + (uint64_t)(u * 2), idesc, acc);
                        acc = 1;
                    }
                    tc_commit(bar_empty + 8 * s);
                }
                if (ok) tc_commit(bar_tfull + 8 * b);
            }
            if (!ok) {
                tc_commit(bar_drain);
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(bar_drain, 0) && global_ns() - t0 < WAIT_LIMIT_NS) {
                }
            }
        }
        __syncwarp();
    } else {
        // ---- epilogue
        dk_wait_prerequisites();
        const int q = warp & 3, e = threadIdx.x - 64, np = g.np, pitch = np + 1, token = e % np, part = e / np, parts = 128 / np;
        const int active = min(g.T, max(0, *g.h.active));
        const bool on = token < active;
        const int target = on ? g.h.targets[token] : -1;
        for (int j = 0; j < mine; ++j) {
            const int tile = (int)blockIdx.x + j * (int)gridDim.x, c0 = tile * HF_COLS, cols = min(HF_COLS, g.V - c0);
            const uint32_t b = j & 1;
            bool ok = mbar_wait(bar_tfull + 8 * b, (uint32_t)(j >> 1) & 1u, abort_word, 74);
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
                tc_fence_after();
                for (int c = 0; c < np; c += 16) {
                    uint32_t v[16];
                    hf_ld_32x16(tmem_base + ((uint32_t)(q * 32) << 16) + b * 64 + c, v);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) s_tile[(q * 32 + lane) * pitch + c + i] = __uint_as_float(v[i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_tempty + 8 * b);
            } else if (lane == 0) {
                s_bad = 1;
            }
            hf_sync();
            if (s_bad) break;
            // np of the tile's columns for the thread's token
            float* const col = s_tile + part * np * pitch + token;
            const int n = max(0, min(np, cols - part * np)), t = target - c0 - part * np;       // the target's place among them
            float m = -INFINITY;
            for (int i = 0; i < np; i += 8) {       // (eight reads on their way; what lies behind the vocabulary is not used)
                float z[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) z[u] = col[(i + u) * pitch];
#pragma unroll
                for (int u = 0; u < 8; ++u) m = i + u < n ? fmaxf(m, z[u]) : m;
            }
            s_max[e] = m;
            hf_sync();
            for (int p = 0; p < parts; ++p) m = fmaxf(m, s_max[p * np + token]);
            const float ref = m == -INFINITY ? 0.f : m * g.h.k2;
            float sum = 0.f;
            if (t >= 0 && t < n) g.h.target_logit[token] = col[t * pitch] * g.h.k2;
            for (int i = 0; i < np; i += 8) {
                float z[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) z[u] = col[(i + u) * pitch];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    float x;
                    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(fmaf(z[u], g.h.k2, -ref)));
                    x = i + u < n && i + u != t ? x : 0.f;
                    sum += x;
                    if (g.h.keep) col[(i + u) * pitch] = x;
                }
            }
            s_sum[e] = sum;
            hf_sync();
            if (part == 0 && on) {
                for (int p = 1; p < parts; ++p) sum += s_sum[p * np + token];
                g.h.part[(size_t)token * g.h.part_ld + tile] = make_float2(ref, sum);
            }
            if (g.h.keep) {         // eight columns of a token per store
                for (int i = part; i < (cols + 7) / 8; i += parts) {
                    uint32_t o[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int c = i * 8 + 2 * u;
                        __nv_bfloat162 p = __floats2bfloat162_rn(c < cols ? s_tile[c * pitch + token] : 0.f, c + 1 < cols ? s_tile[(c + 1) * pitch + token] : 0.f);
                        o[u] = *reinterpret_cast<uint32_t*>(&p);
                    }
                    if (on) *reinterpret_cast<uint4*>(g.E + (size_t)token * g.lde + c0 + i * 8) = make_uint4(o[0], o[1], o[2], o[3]);
                }
                hf_sync();          // before the next tile is written there
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    if (threadIdx.x == 0 && *abort_word != 0) {
        if (atomicCAS(g.status, 0, DEV_TIMEOUT) == 0) g.status[1] = *abort_word * 1000000 + (int)blockIdx.x;
    }
}

}  // namespace sm100

marlaas_status_t launch_head_few(const marlaas_pool* pool, int64_t T, int64_t d, int64_t V, const bf16* rows, int64_t dp, const bf16* W, int64_t ldw,
                                 bf16* E, int64_t lde, const HeadEpilogue& h, cudaStream_t st) {
    using namespace sm100;
    HeadFewArgs g;
    memset(&g, 0, sizeof(g));
    g.T = (int)T;
    g.V = (int)V;
    g.np = T <= 16 ? 16 : T <= 32 ? 32 : 64;
    g.nkb = (int)cdiv(d, 64);
    g.tiles = (int)cdiv(V, HF_COLS);
    g.E = E;
    g.lde = lde;
    g.h = h;
    g.status = pool->d_status;
    alignas(64) CUtensorMap tmW, tmX;
    marlaas_status_t rc;
    if ((rc = make_map(&tmW, W, d, V, ldw, 64, 64)) != MARLAAS_OK) return rc;
    if ((rc = make_map(&tmX, rows, T, dp, dp, 64, (uint32_t)g.np)) != MARLAAS_OK) return rc;
    static bool attr_set[64] = {};
    if (pool->device >= 64 || !attr_set[pool->device]) {
        MARLAAS_CUDA_TRY(cudaFuncSetAttribute(k_head_few, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)HF_SMEM));
        if (pool->device < 64) attr_set[pool->device] = true;
    }
    return launch_link("k_head_few", k_head_few, dim3((unsigned)(g.tiles < pool->sm_count ? g.tiles : pool->sm_count)), HF_THREADS, HF_SMEM, true, st,
                       tmW, tmX, g);        // (behind the gathering kernel)
}

}  // namespace marlaas
