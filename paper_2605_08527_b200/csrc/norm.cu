// Layer norm and RMS norm whose gain and bias are each tenant's own, forward and backward (a norm in front of an adapted
// projection; its parameters are trained beside the adapters).  For token i of tenant t, over the d elements of its row:
//     xh = (x - mean) rstd,   rstd = 1 / sqrt(var + eps)          y = xh gain_t + bias_t
//     a = dy gain_t           dx = rstd (a - avg(a) - xh avg(a xh))
//     dgain_t = sum over its tokens of dy xh                      dbias_t = sum of dy
// (RMS norm: mean = 0 and no avg(a).)  Statistics and sums are fp32; x, y, dy, dx are bf16, rounded once when they are written.
// Both passes are bound by HBM: 4 bytes per element forward, 6 backward.
#include <string.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "sm100_cluster.cuh"

namespace marlaas {
using sm100::dk_report;

struct NormArgs {
    int64_t T;
    int d, S, cap;
    const int32_t* off;
    const int32_t* slot;
    const bf16* x; int64_t ldx;
    const bf16* dy; int64_t lddy;
    bf16* y; int64_t ldy;               // forward: y, backward: dx (or NULL)
    const float* gain;                  // [cap + 1][d]
    const float* bias;                  // [cap + 1][d] or NULL
    float eps;
    float* mean; float* rstd;           // forward: outputs, each may be NULL
    const float* mean_in; const float* rstd_in;
    // backward: tokens in the order of their tenants, and the partial sums of the runs
    const int32_t* perm;
    const int32_t* key_off;             // [cap + 2]
    float* partial;                     // [groups + cap + 1][2][d]
    int64_t rows_per_group;
    float* dgain; float* dbias;         // [cap + 1][d], each may be NULL
    int accumulate;
    int32_t* status;
};

__device__ __forceinline__ void unpack8(const uint4& q, float (&f)[8]) {
    const uint32_t* w = &q.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    uint4 q;
    uint32_t* w = &q.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t*>(&p);
    }
    return q;
}
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---- forward ----
// W warps per row, NV vectors of 8 elements per lane, the row in registers between its statistics and the output.
constexpr int NORM_THREADS = 256;
template <int W, int NV, bool RMS>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_forward(const NormArgs a) {
    constexpr int ROWS = NORM_THREADS / 32 / W;
    __shared__ float s_part[2][ROWS][W];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = warp / W, wg = warp % W, l = wg * 32 + lane;
    const int nvec = a.d / 8;
    const float inv_d = 1.f / (float)a.d;
    for (int64_t s = (int64_t)blockIdx.x * NORM_THREADS + threadIdx.x; s < a.S; s += (int64_t)gridDim.x * NORM_THREADS) {
        const int p = a.off[s], q = a.off[s + 1], t = a.slot[s];
        if (q < p || p < 0 || q > a.T || (s == 0 && p != 0) || (s == a.S - 1 && q != a.T)) dk_report(a.status, DEV_BAD_TABLE, (int)s);
        if (t < -1 || t >= a.cap) dk_report(a.status, DEV_BAD_INDEX, (int)s);
    }
    // sum over the row's lanes; all threads of the CTA take the same steps
    auto row_sum = [&](float v, int which) {
        v = warp_sum(v);
        if (W == 1) return v;
        if (lane == 0) s_part[which][g][wg] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += s_part[which][g][w];
        return v;
    };
    for (int64_t i0 = (int64_t)blockIdx.x * ROWS; i0 < a.T; i0 += (int64_t)gridDim.x * ROWS) {
        const int64_t i = i0 + g;
        const bool on = i < a.T;
        uint4 q[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = l + j * 32 * W;
            q[j] = on && v < nvec ? reinterpret_cast<const uint4*>(a.x + i * a.ldx)[v] : make_uint4(0u, 0u, 0u, 0u);
        }
        int lo = 0, hi = on ? a.S : 0;          // the token's segment, while the row is on its way
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(a.off + mid + 1) > i) hi = mid; else lo = mid + 1;
        }
        int t = on && lo < a.S ? a.slot[lo] : -1;
        if (t < 0 || t >= a.cap) t = a.cap;
        const float* gain = a.gain + (size_t)t * a.d;
        const float* bias = a.bias ? a.bias + (size_t)t * a.d : nullptr;
        float mean = 0.f, f[8];
        if (!RMS) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                unpack8(q[j], f);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += f[e];
            }
            mean = row_sum(sum, 0) * inv_d;
        }
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (l + j * 32 * W < nvec) {
                unpack8(q[j], f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float c = f[e] - mean;
                    sq = fmaf(c, c, sq);
                }
            }
        }
        const float rstd = 1.f / sqrtf(fmaf(row_sum(sq, 1), inv_d, a.eps));
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = l + j * 32 * W;
            if (on && v < nvec) {
                float w[8];
                unpack8(q[j], f);
                load8(gain + v * 8, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean) * rstd * w[e];
                if (bias) {
                    load8(bias + v * 8, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] += w[e];
                }
                reinterpret_cast<uint4*>(a.y + i * a.ldy)[v] = pack8(f);
            }
        }
        if (on && l == 0) {
            if (a.mean) a.mean[i] = mean;
            if (a.rstd) a.rstd[i] = rstd;
        }
        if (W > 1) __syncthreads();
    }
}

// ---- backward ----
// A group of W warps takes a run of the ordered tokens, one row after another; a thread keeps the same NV x 8 columns
// throughout, so that the tenant's gain and the sums for dgain and dbias stay in its registers until the tenant changes.  Rows
// are fetched DEPTH - 1 ahead by asynchronous copies into shared memory that only the fetching thread reads: no barrier but the one
// for a row's two sums.  The sums of a (group, tenant) pair go to partial[group + tenant]: both only rise along the ordered
// tokens, so no two pairs share a place, and the order of all additions depends on the sizes and the tables alone.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
constexpr int NORM_BACK_THREADS = 512;

template <int NV, int NORM_DEPTH, bool RMS>
__global__ void __launch_bounds__(NORM_BACK_THREADS) k_norm_backward(const NormArgs a, int W, int G) {
    extern __shared__ uint4 s_ring[];       // [DEPTH][2][NV][threads]
    __shared__ float2 s_part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = warp / W, wg = warp % W, l = wg * 32 + lane;
    const int nvec = a.d / 8, threads = blockDim.x;
    const float inv_d = 1.f / (float)a.d;
    const int64_t q = (int64_t)blockIdx.x * G + g;
    const int64_t p0 = q * a.rows_per_group, p1 = p0 + a.rows_per_group < a.T ? p0 + a.rows_per_group : a.T;
    if (p0 >= a.T) return;                  // (a group synchronises with itself alone)
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + threadIdx.x * 16;
    auto fetch = [&](int64_t p) -> int64_t {        // starts row p's copies; its token
        int64_t i = -1;
        if (p < p1) {
            i = a.perm[p];
            const int st = (int)((p - p0) % NORM_DEPTH);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int v = l + j * 32 * W;
                if (v < nvec) {
                    copy16(ring + ((st * 2 + 0) * NV + j) * threads * 16, a.x + i * a.ldx + v * 8);
                    copy16(ring + ((st * 2 + 1) * NV + j) * threads * 16, a.dy + i * a.lddy + v * 8);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return i;
    };
    int64_t tok[NORM_DEPTH];
#pragma unroll
    for (int u = 0; u < NORM_DEPTH - 1; ++u) tok[u] = fetch(p0 + u);
    int key = -1;
    int64_t key_end = p0;
    float gain[NV][8], sg[NV][8], sb[NV][8];
    auto flush = [&]() {
        float* out = a.partial + (size_t)(q + key) * 2 * a.d;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = l + j * 32 * W;
            if (v < nvec) {
                float4* o = reinterpret_cast<float4*>(out + v * 8);
                o[0] = make_float4(sg[j][0], sg[j][1], sg[j][2], sg[j][3]);
                o[1] = make_float4(sg[j][4], sg[j][5], sg[j][6], sg[j][7]);
                if (a.dbias) {
                    o = reinterpret_cast<float4*>(out + a.d + v * 8);
                    o[0] = make_float4(sb[j][0], sb[j][1], sb[j][2], sb[j][3]);
                    o[1] = make_float4(sb[j][4], sb[j][5], sb[j][6], sb[j][7]);
                }
            }
        }
    };
    int par = 0;
    for (int64_t pb = p0; pb < p1; pb += NORM_DEPTH) {
#pragma unroll
        for (int u = 0; u < NORM_DEPTH; ++u) {
            const int64_t p = pb + u;
            if (p >= p1) break;
            tok[(u + NORM_DEPTH - 1) % NORM_DEPTH] = fetch(p + NORM_DEPTH - 1);
            const int64_t i = tok[u];
            const float mean = RMS ? 0.f : a.mean_in[i], rstd = a.rstd_in[i];
            if (p >= key_end) {             // the next tenant that has tokens
                if (key >= 0) flush();
                do key_end = a.key_off[++key + 1]; while (key_end <= p);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int v = l + j * 32 * W;
                    if (v < nvec) load8(a.gain + (size_t)key * a.d + v * 8, gain[j]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sg[j][e] = sb[j][e] = 0.f;
                }
            }
            asm volatile("cp.async.wait_group %0;" ::"n"(NORM_DEPTH - 1) : "memory");
            const int st = u;
            float2 sum = make_float2(0.f, 0.f);
            float xh[NV][8], av[NV][8];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (l + j * 32 * W < nvec) {
                    float dy[8];
                    unpack8(s_ring[((st * 2 + 0) * NV + j) * threads + threadIdx.x], xh[j]);
                    unpack8(s_ring[((st * 2 + 1) * NV + j) * threads + threadIdx.x], dy);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        xh[j][e] = (xh[j][e] - mean) * rstd;
                        av[j][e] = dy[e] * gain[j][e];
                        sg[j][e] = fmaf(dy[e], xh[j][e], sg[j][e]);
                        sb[j][e] += dy[e];
                        if (!RMS) sum.x += av[j][e];
                        sum.y = fmaf(av[j][e], xh[j][e], sum.y);
                    }
                }
            }
            if (a.y) {
                if (!RMS) sum.x = warp_sum(sum.x);
                sum.y = warp_sum(sum.y);
                if (W > 1) {
                    if (lane == 0) s_part[par][warp] = sum;
                    asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "r"(32 * W) : "memory");
                    sum = make_float2(0.f, 0.f);
                    for (int w = 0; w < W; ++w) {
                        const float2 o = s_part[par][g * W + w];
                        sum.x += o.x;
                        sum.y += o.y;
                    }
                    par ^= 1;
                }
                const float ma = sum.x * inv_d, mx = sum.y * inv_d;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int v = l + j * 32 * W;
                    if (v < nvec) {
                        float o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = rstd * (av[j][e] - ma - xh[j][e] * mx);
                        reinterpret_cast<uint4*>(a.y + i * a.ldy)[v] = pack8(o);
                    }
                }
            }
        }
    }
    if (a.partial) flush();
}

// dgain and dbias of one tenant, 32 columns per CTA: eight warps share the tenant's partial sums, then a fixed tree.
__global__ void __launch_bounds__(256) k_norm_reduce(const NormArgs a) {
    __shared__ float s_sum[8][2][32];
    const int key = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const int64_t b = a.key_off[key], e = a.key_off[key + 1];
    const bool on = c < a.d;
    float g = 0.f, h = 0.f;
    if (e > b && on) {
        const int64_t q1 = (e - 1) / a.rows_per_group;
        for (int64_t q = b / a.rows_per_group + warp; q <= q1; q += 8) {
            const float* in = a.partial + (size_t)(q + key) * 2 * a.d + c;
            g += in[0];
            if (a.dbias) h += in[a.d];
        }
    }
    s_sum[warp][0][lane] = g;
    s_sum[warp][1][lane] = h;
    __syncthreads();
    if (warp >= 2 || !on) return;
    float* out = warp == 0 ? a.dgain : a.dbias;
    if (!out) return;
    out += (size_t)key * a.d + c;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += s_sum[w][warp][lane];
    *out = a.accumulate ? *out + v : v;
}

// How the backward pass cuts a batch: warps per row and rows of a CTA at a time, groups in all.
struct NormPlan {
    int NV, W, G;
    int64_t groups, rows;
};
static NormPlan norm_plan(const marlaas_pool* pool, int64_t T, int d) {
    NormPlan p;
    const int nvec = d / 8;
    p.NV = 1;
    while (p.NV * NORM_BACK_THREADS < nvec) p.NV *= 2;           // one vector per lane while 16 warps hold a row
    p.W = (int)cdiv(nvec, 32 * p.NV);
    p.G = std::min(8, NORM_BACK_THREADS / 32 / p.W);
    const int64_t most = (int64_t)pool->sm_count * 2 * p.G;      // two CTAs per SM
    p.rows = std::max<int64_t>(cdiv(T, most), 1);
    p.groups = cdiv(cdiv(T, p.rows), p.G) * p.G;
    return p;
}

struct NormWorkspace {
    int32_t* off;           // [S + 1] host tables
    int32_t* slot;          // [S]
    int32_t* perm;          // [T]
    int32_t* key_off;       // [cap + 2]
    int32_t* scratch;
    float* partial;
    size_t total_bytes;
};
static NormWorkspace carve_norm(const marlaas_pool* pool, int64_t T, int32_t S, int64_t d, bool backward, void* base) {
    NormWorkspace w;
    memset(&w, 0, sizeof(w));
    char* p = (char*)base;
    size_t o = 0;
    auto take = [&](size_t bytes) { char* q = p ? p + o : nullptr; o += align_up(bytes, 256); return q; };
    w.off = (int32_t*)take(sizeof(int32_t) * ((size_t)S + 1));
    w.slot = (int32_t*)take(sizeof(int32_t) * (size_t)S);
    if (backward) {
        const NormPlan n = norm_plan(pool, T, (int)d);
        w.perm = (int32_t*)take(sizeof(int32_t) * (size_t)T);
        w.key_off = (int32_t*)take(sizeof(int32_t) * ((size_t)pool->cap + 2));
        w.scratch = (int32_t*)take(sizeof(int32_t) * order_scratch_ints(T, pool->cap + 1));
        w.partial = (float*)take(sizeof(float) * (size_t)(n.groups + pool->cap + 1) * 2 * (size_t)d);
    }
    w.total_bytes = o;
    return w;
}

static marlaas_status_t launch_norm_forward(const marlaas_pool* pool, const NormArgs& a, bool rms, cudaStream_t st) {
    const int nvec = a.d / 8;
    // One warp per row while its registers hold it and there are rows enough for two CTAs per SM; else four.
    const int W = nvec <= 16 * 32 && cdiv(a.T, 8) >= 2 * (int64_t)pool->sm_count ? 1 : 4;
    int NV = 1;
    while (NV * 32 * W < nvec) NV *= 2;
    const int rows = NORM_THREADS / 32 / W;
    const unsigned grid = (unsigned)std::min<int64_t>(cdiv(a.T, rows), (int64_t)pool->sm_count * 8);
#define NORM_GO(w, n)                                                                   \
    if (W == w && NV == n) {                                                            \
        if (rms) k_norm_forward<w, n, true><<<grid, NORM_THREADS, 0, st>>>(a);          \
        else k_norm_forward<w, n, false><<<grid, NORM_THREADS, 0, st>>>(a);             \
    }
    NORM_GO(1, 1) NORM_GO(1, 2) NORM_GO(1, 4) NORM_GO(1, 8) NORM_GO(1, 16)
    NORM_GO(4, 1) NORM_GO(4, 2) NORM_GO(4, 4) NORM_GO(4, 8) NORM_GO(4, 16)
#undef NORM_GO
    MARLAAS_LAUNCH_CHECK("k_norm_forward");
    return MARLAAS_OK;
}

template <int NV, bool RMS>
static marlaas_status_t launch_norm_backward_t(const marlaas_pool* pool, const NormArgs& a, const NormPlan& n, cudaStream_t st) {
    constexpr int DEPTH = NV == 4 ? 2 : 4;          // as deep as shared memory allows for the widest rows
    constexpr size_t most = (size_t)DEPTH * 2 * NV * NORM_BACK_THREADS * 16;
    const int threads = 32 * n.W * n.G;
    static bool attr_set[64] = {};
    if (pool->device >= 64 || !attr_set[pool->device]) {
        MARLAAS_CUDA_TRY(cudaFuncSetAttribute(k_norm_backward<NV, DEPTH, RMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
        if (pool->device < 64) attr_set[pool->device] = true;
    }
    k_norm_backward<NV, DEPTH, RMS><<<(unsigned)(n.groups / n.G), threads, (size_t)DEPTH * 2 * NV * threads * 16, st>>>(a, n.W, n.G);
    MARLAAS_LAUNCH_CHECK("k_norm_backward");
    return MARLAAS_OK;
}

static bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// An output matrix may be an input matrix itself, with the same leading dimension; any other overlap is refused.
static marlaas_status_t check_overlap(const char* fn, const char* name, const void* out, int64_t ldo, const void* in, int64_t ldi,
                                      int64_t T, int64_t d) {
    const uintptr_t a0 = (uintptr_t)out, a1 = a0 + 2 * (size_t)((T - 1) * ldo + d), b0 = (uintptr_t)in, b1 = b0 + 2 * (size_t)((T - 1) * ldi + d);
    if (a0 < b1 && b0 < a1 && !(a0 == b0 && ldo == ldi))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: %s overlaps an input without being the same matrix", fn, name);
    return MARLAAS_OK;
}

// What both passes check, and the table's place on the device.
static marlaas_status_t check_norm(const char* fn, const marlaas_pool* pool, int64_t T, int64_t d, const marlaas_segments_t* seg,
                                   const float* gain, const float* bias, uint32_t flags, uint32_t allowed) {
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (T < 0 || T >= (1ll << 31)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: T out of range", fn);
    if (d < 8 || d > MARLAAS_MAX_NORM_WIDTH || d % 8 != 0)
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: width %lld must be a multiple of 8 from 8 to %d", fn, (long long)d, (int)MARLAAS_MAX_NORM_WIDTH);
    if (flags & ~allowed) return fail(MARLAAS_ERR_INVALID_ARG, "%s: a flag does not apply to this call", fn);
    if (!gain || misaligned(gain, 16) || misaligned(bias, 16))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: gain is NULL, or gain or bias is not 16-byte aligned", fn);
    return check_segments(fn, pool, T, seg, flags, nullptr);
}

static marlaas_status_t stage_table(const marlaas_segments_t* seg, const NormWorkspace& ws, NormArgs* a, cudaStream_t st) {
    // the copy's source is the call's own and pageable: staged when the copy returns
    const size_t S = (size_t)seg->num_segments;
    std::vector<int32_t> copy((size_t)(ws.slot - ws.off) + S);
    std::copy(seg->seg_offsets, seg->seg_offsets + S + 1, copy.begin());
    std::copy(seg->seg_slot, seg->seg_slot + S, copy.begin() + (ws.slot - ws.off));
    MARLAAS_CUDA_TRY(cudaMemcpyAsync(ws.off, copy.data(), sizeof(int32_t) * copy.size(), cudaMemcpyHostToDevice, st));
    a->off = ws.off;
    a->slot = ws.slot;
    return MARLAAS_OK;
}

}  // namespace marlaas

using namespace marlaas;

extern "C" {

size_t marlaas_layer_norm_workspace_bytes(const marlaas_pool_t* pool, int64_t T, int64_t d, int32_t num_segments, int32_t backward) {
    if (!pool || T < 0 || T >= (1ll << 31) || num_segments < 0 || num_segments > MAX_SEGMENTS || d < 8 || d > MARLAAS_MAX_NORM_WIDTH || d % 8 != 0)
        return 0;
    return carve_norm(pool, T, num_segments, d, backward != 0, nullptr).total_bytes;
}

marlaas_status_t marlaas_layer_norm(marlaas_pool_t* pool, int64_t T, int64_t d, const void* x, int64_t ldx,
                                            const marlaas_segments_t* seg, const float* gain, const float* bias, float eps, void* y,
                                            int64_t ldy, float* mean, float* rstd, void* workspace, size_t workspace_bytes,
                                            uint32_t flags, void* cuda_stream) try {
    const char* fn = "layer_norm";
    marlaas_status_t rc = check_norm(fn, pool, T, d, seg, gain, bias, flags,
                                     MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC | MARLAAS_FLAG_RMS_NORM);
    if (rc != MARLAAS_OK) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: eps must be finite and not negative", fn);
    if (misaligned(mean, 4) || misaligned(rstd, 4)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: an output is misaligned", fn);
    if (T == 0) return MARLAAS_OK;
    if ((rc = check_matrix(fn, "x", x, ldx, d)) != MARLAAS_OK) return rc;
    if ((rc = check_matrix(fn, "y", y, ldy, d)) != MARLAAS_OK) return rc;
    if ((rc = check_overlap(fn, "y", y, ldy, x, ldx, T, d)) != MARLAAS_OK) return rc;
    const bool host = (flags & MARLAAS_FLAG_HOST_TABLE) != 0;
    if (host && (!workspace || misaligned(workspace, 256))) return fail(MARLAAS_ERR_INVALID_ARG, "%s: workspace NULL or misaligned", fn);
    const NormWorkspace ws = carve_norm(pool, T, seg->num_segments, d, false, workspace);
    if (host && workspace_bytes < ws.total_bytes)
        return fail(MARLAAS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < required %zu", fn, workspace_bytes, ws.total_bytes);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    NormArgs a;
    memset(&a, 0, sizeof(a));
    a.T = T; a.d = (int)d; a.S = seg->num_segments; a.cap = pool->cap;
    a.off = seg->seg_offsets; a.slot = seg->seg_slot;
    a.x = (const bf16*)x; a.ldx = ldx; a.y = (bf16*)y; a.ldy = ldy;
    a.gain = gain; a.bias = bias; a.eps = eps; a.mean = mean; a.rstd = rstd; a.status = pool->d_status;
    if (host && (rc = stage_table(seg, ws, &a, st)) != MARLAAS_OK) return rc;
    if ((rc = launch_norm_forward(pool, a, (flags & MARLAAS_FLAG_RMS_NORM) != 0, st)) != MARLAAS_OK) return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "layer_norm: %s", e.what());
}

marlaas_status_t marlaas_layer_norm_backward(marlaas_pool_t* pool, int64_t T, int64_t d, const void* x, int64_t ldx, const void* dy,
                                             int64_t lddy, const marlaas_segments_t* seg, const float* gain, const float* mean,
                                             const float* rstd, void* dx, int64_t lddx, float* dgain, float* dbias, void* workspace,
                                             size_t workspace_bytes, uint32_t flags, void* cuda_stream) try {
    const char* fn = "layer_norm_backward";
    marlaas_status_t rc = check_norm(fn, pool, T, d, seg, gain, nullptr, flags,
                                     MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC | MARLAAS_FLAG_RMS_NORM | MARLAAS_FLAG_ACCUMULATE);
    if (rc != MARLAAS_OK) return rc;
    const bool rms = (flags & MARLAAS_FLAG_RMS_NORM) != 0, host = (flags & MARLAAS_FLAG_HOST_TABLE) != 0;
    const bool accumulate = (flags & MARLAAS_FLAG_ACCUMULATE) != 0;
    if (misaligned(dgain, 16) || misaligned(dbias, 16)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: dgain or dbias is not 16-byte aligned", fn);
    if (!dx && !dgain && !dbias) return fail(MARLAAS_ERR_INVALID_ARG, "%s: no output", fn);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (T == 0) {
        MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
        const size_t bytes = sizeof(float) * ((size_t)pool->cap + 1) * (size_t)d;
        if (dgain && !accumulate) MARLAAS_CUDA_TRY(cudaMemsetAsync(dgain, 0, bytes, st));
        if (dbias && !accumulate) MARLAAS_CUDA_TRY(cudaMemsetAsync(dbias, 0, bytes, st));
        return finish(pool, flags, st);
    }
    if ((rc = check_matrix(fn, "x", x, ldx, d)) != MARLAAS_OK) return rc;
    if ((rc = check_matrix(fn, "dy", dy, lddy, d)) != MARLAAS_OK) return rc;
    if (dx) {
        if ((rc = check_matrix(fn, "dx", dx, lddx, d)) != MARLAAS_OK) return rc;
        if ((rc = check_overlap(fn, "dx", dx, lddx, x, ldx, T, d)) != MARLAAS_OK) return rc;
        if ((rc = check_overlap(fn, "dx", dx, lddx, dy, lddy, T, d)) != MARLAAS_OK) return rc;
    }
    if (!rstd || misaligned(rstd, 4) || (!rms && !mean) || misaligned(mean, 4))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: mean or rstd is NULL or misaligned", fn);
    if (!workspace || misaligned(workspace, 256)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: workspace NULL or misaligned", fn);
    const NormWorkspace ws = carve_norm(pool, T, seg->num_segments, d, true, workspace);
    if (workspace_bytes < ws.total_bytes)
        return fail(MARLAAS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < required %zu", fn, workspace_bytes, ws.total_bytes);
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    const NormPlan n = norm_plan(pool, T, (int)d);
    NormArgs a;
    memset(&a, 0, sizeof(a));
    a.T = T; a.d = (int)d; a.S = seg->num_segments; a.cap = pool->cap;
    a.off = seg->seg_offsets; a.slot = seg->seg_slot;
    a.x = (const bf16*)x; a.ldx = ldx; a.dy = (const bf16*)dy; a.lddy = lddy; a.y = (bf16*)dx; a.ldy = lddx;
    a.gain = gain; a.mean_in = mean; a.rstd_in = rstd; a.status = pool->d_status;
    a.perm = ws.perm; a.key_off = ws.key_off; a.rows_per_group = n.rows;
    a.partial = dgain || dbias ? ws.partial : nullptr;
    a.dgain = dgain; a.dbias = dbias; a.accumulate = accumulate ? 1 : 0;
    if (host && (rc = stage_table(seg, ws, &a, st)) != MARLAAS_OK) return rc;
    OrderArgs o;
    memset(&o, 0, sizeof(o));
    o.T = T; o.S = a.S; o.off = a.off; o.slot = a.slot; o.cap = pool->cap; o.nkeys = pool->cap + 1;
    o.perm = ws.perm; o.key_off = ws.key_off;
    if ((rc = launch_order(pool, o, ws.scratch, st)) != MARLAAS_OK) return rc;
    if (n.NV == 1) rc = rms ? launch_norm_backward_t<1, true>(pool, a, n, st) : launch_norm_backward_t<1, false>(pool, a, n, st);
    else if (n.NV == 2) rc = rms ? launch_norm_backward_t<2, true>(pool, a, n, st) : launch_norm_backward_t<2, false>(pool, a, n, st);
    else rc = rms ? launch_norm_backward_t<4, true>(pool, a, n, st) : launch_norm_backward_t<4, false>(pool, a, n, st);
    if (rc != MARLAAS_OK) return rc;
    if (a.partial) {
        k_norm_reduce<<<dim3((unsigned)cdiv(d, 32), (unsigned)(pool->cap + 1)), 256, 0, st>>>(a);
        MARLAAS_LAUNCH_CHECK("k_norm_reduce");
    }
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "layer_norm_backward: %s", e.what());
}

}  // extern "C"
