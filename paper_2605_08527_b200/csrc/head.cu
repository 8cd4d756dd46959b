// Cross entropy of the vocabulary head from the last hidden states: log-probabilities, loss and the gradient by the hidden
// states, without logits in memory (Algorithm 1, training branch: what the policy update of a batch starts from).  With
// k = inv_temperature, for a token i that counts (target y >= 0, weight w != 0):
//     z = k x_i W        logp = z_y - log sum exp z        loss = sum_i w_i (-logp_i)
//     dx_i = grad_scale k w_i (p - e_y) W^T,   p = softmax(z)
// W is frozen, there is no dW.  Two products of 2 T d V operations, one without the gradient:
//   1. the tokens that count are gathered, in their order, so that ignored ones (prompts, padding) cost nothing
//   2. x W tile by tile in tensor memory (a few tokens: head_few.cu); a tile leaves it as a pair (reference, sum of exponentials) per row, and for the
//      gradient as exponentials in bf16, relative to the row's reference in the tile: their error is 2^-8 of each probability,
//      where rounding the logits would make it 2^-8 of a logit
//   3. a row's pairs give the sum R of the exponentials of all entries but the target, and logp = -log(1 + R / exp z_y), which
//      keeps its digits however sure the model is; the exponentials become p - e_y in place
//   4. times W^T, cut along the vocabulary so that few rows fill the SMs too; the row's factor enters in fp32
// The exponentials of at most HEAD_PIECE_BYTES are held at a time: larger batches go through steps 2 to 4 in pieces of rows.
// The tensor cores bound it: at 2048 counted rows x 131072 x 4096 steps 2 and 4 take 1.67 and 1.66 ms, 1.32 PFLOP/s each, and step
// 3 0.19 ms, which is the exponentials once from HBM and back.  Few rows are bound by W's bytes and by latency: 32 x 1024 x 32768
// without gradient 27 us in four dependent kernels, of which W's 67 MB are 10.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "sm100_cluster.cuh"

namespace marlaas {
using sm100::dk_report;

constexpr size_t HEAD_PIECE_BYTES = (size_t)512 << 20;
constexpr int HEAD_ITEMS = 768;             // tiles of partial gradients, 256 KB each
constexpr int HEAD_THREADS = 256;
constexpr float HEAD_LOG2E = 1.4426950408889634f, HEAD_LN2 = 0.6931471805599453f;

struct HeadArgs {
    int64_t T;
    int d, V, NT;                           // NT: tiles of the vocabulary, of 256 columns, or 128 for a few tokens
    int tile_shift;                         // log2 of a tile's vectors of eight columns
    int dp;                                 // d in whole 64-element panels: the pitch of the rows
    const bf16* x; int64_t ldx;
    const int32_t* targets;
    const float* weight;                    // or NULL
    float factor;                           // grad_scale * inv_temperature
    const int32_t* perm;
    const int32_t* active;
    bf16* rows;                             // [T][dp] the tokens that count, zeros behind each
    int32_t* row_target;                    // [T]
    float* row_coef;                        // [T]
    bf16* E; int64_t lde;
    float2* part;
    float* target_logit;                    // [piece] in units of log 2
    float4* terms;                          // [T] or NULL
    float* logp;                            // [T] or NULL
    bf16* dx; int64_t lddx;                 // or NULL
};

// A token that counts is copied to its row, of another one the outputs are cleared; a warp per place in the order.  Batches of at
// most HEAD_SMALL_T tokens need no order made before (SMALL): a warp takes a token, and each CTA counts the tokens before its own,
// which costs tokens^2 / 2048 loads where the order costs three kernels (whole calls, V = 1000, d = 1024, counted here and ordered
// before: 1024 tokens 25 and 29 us, 4096 37 and 42, 8192 65 and 66, 16384 117 and 109).
constexpr int HEAD_SMALL_T = 4096;
template <bool SMALL>
__global__ void __launch_bounds__(HEAD_THREADS) k_head_gather(const HeadArgs a, int32_t* perm, int32_t* active, int32_t* status) {
    __shared__ int s_cnt[HEAD_THREADS / 32], s_on[HEAD_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    sm100::dk_launch_dependents();
    int64_t p = (int64_t)blockIdx.x * (HEAD_THREADS / 32) + warp, i = p;
    bool on;
    if (SMALL) {
        auto counts = [&](int64_t j) {
            const int y = a.targets[j];
            return y >= 0 && y < a.V && !(a.weight && a.weight[j] == 0.f);
        };
        const int64_t first = (int64_t)blockIdx.x * (HEAD_THREADS / 32);
        int n = 0;
        for (int64_t j = threadIdx.x; j < first; j += HEAD_THREADS) n += counts(j);
        for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        on = i < a.T && counts(i);
        if (lane == 0) {
            s_cnt[warp] = n;
            s_on[warp] = on;
            if (i < a.T && a.targets[i] >= a.V) dk_report(status, DEV_BAD_INDEX, (int)i);
        }
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < HEAD_THREADS / 32; ++w) {
            before += s_cnt[w] + (w < warp ? s_on[w] : 0);
            all += s_cnt[w] + s_on[w];
        }
        if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *active = all;
        if (on && lane == 0) perm[before] = (int)i;
        p = before;
    } else {
        on = p < *active;
        if (p < a.T) i = perm[p];
    }
    if (i >= a.T) return;
    const int nvec = a.d / 8;
    if (on) {
        const uint4* src = reinterpret_cast<const uint4*>(a.x + i * a.ldx);
        uint4* dst = reinterpret_cast<uint4*>(a.rows + p * a.dp);
        constexpr int U = 4;                    // vectors on their way per lane
        for (int v0 = lane; v0 < a.dp / 8; v0 += 32 * U) {
            uint4 q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) q[u] = v0 + 32 * u < nvec ? src[v0 + 32 * u] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v0 + 32 * u < a.dp / 8) dst[v0 + 32 * u] = q[u];
        }
        if (lane == 0) {
            a.row_target[p] = a.targets[i];
            a.row_coef[p] = a.factor * (a.weight ? a.weight[i] : 1.f);
        }
        return;
    }
    if (a.dx) {
        uint4* dst = reinterpret_cast<uint4*>(a.dx + i * a.lddx);
        for (int v = lane; v < nvec; v += 32) dst[v] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (lane == 0) {
        if (a.logp) a.logp[i] = 0.f;
        if (a.terms) a.terms[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
}

// One CTA per row of the piece: log-sum-exp of the tiles' pairs, the token's outputs, and p - e_y in place of the exponentials.
// Streams 4 bytes per element: HBM.
template <bool GRAD>
__global__ void __launch_bounds__(HEAD_THREADS) k_head_rows(const HeadArgs a, int row0) {
    __shared__ float s_f[GRAD ? MARLAAS_MAX_VOCABULARY / 128 : 1];
    __shared__ float s_red[HEAD_THREADS / 32];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    sm100::dk_wait_prerequisites();
    sm100::dk_launch_dependents();
    if (row0 + row >= *a.active) return;
    const float2* part = a.part + (size_t)row * a.NT;
    auto all = [&](float v, bool is_max) {      // the same tree in every call
        for (int o = 16; o > 0; o >>= 1) {
            const float u = __shfl_xor_sync(0xffffffffu, v, o);
            v = is_max ? fmaxf(v, u) : v + u;
        }
        __syncthreads();
        if (lane == 0) s_red[warp] = v;
        __syncthreads();
        v = s_red[0];
        for (int w = 1; w < HEAD_THREADS / 32; ++w) v = is_max ? fmaxf(v, s_red[w]) : v + s_red[w];
        return v;
    };
    float m = -INFINITY;
    for (int j = tid; j < a.NT; j += HEAD_THREADS) m = part[j].y != 0.f ? fmaxf(m, part[j].x) : m;     // (a tile of -inf alone has the sum 0)
    m = all(m, true);
    float s = 0.f;
    for (int j = tid; j < a.NT; j += HEAD_THREADS) {
        const float2 q = part[j];
        s += q.y != 0.f ? q.y * exp2f(q.x - m) : 0.f;
    }
    s = all(s, false);
    // m, s: reference and sum of the others' exponentials; zy, the target's logit, may be anything beside them
    const float zy = a.target_logit[row], top = s == 0.f ? zy : fmaxf(m, zy), gap = m - zy;
    const bool none = s == 0.f && zy == -INFINITY;      // no logit above -inf: no distribution
    float logp = s == 0.f ? zy - zy : gap < 30.f ? -log1pf(s * exp2f(gap)) : -(gap * HEAD_LN2 + logf(s + exp2f(-gap)));
    if (!(zy < INFINITY)) logp = NAN;
    if (none) logp = 0.f;
    if (tid == 0) {
        const int64_t i = a.perm[row0 + row];
        const float w = a.weight ? a.weight[i] : 1.f;
        if (a.logp) a.logp[i] = logp;
        if (a.terms) a.terms[i] = make_float4(-w * logp, w, -logp, 1.f);
    }
    if (!GRAD) return;
    const float inv = none ? 0.f : 1.f / (s * exp2f(s == 0.f ? 0.f : m - top) + exp2f(zy - top));
    for (int j = tid; j < a.NT; j += HEAD_THREADS) {
        const float2 q = part[j];
        s_f[j] = q.y != 0.f ? exp2f(q.x - top) * inv : 0.f;
    }
    __syncthreads();
    const int y = a.row_target[row0 + row], nvec = (a.V + 7) / 8;
    const float py = none ? 0.f : expm1f(logp);
    uint4* e = reinterpret_cast<uint4*>(a.E + (size_t)row * a.lde);
    constexpr int U = 4;                        // vectors on their way per thread
    for (int v0 = tid; v0 < nvec; v0 += HEAD_THREADS * U) {
        uint4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = v0 + u * HEAD_THREADS;
            if (v < nvec) q[u] = e[v];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = v0 + u * HEAD_THREADS;
            if (v >= nvec) break;
            uint32_t* w = &q[u].x;
            const float f = s_f[v >> a.tile_shift];
            const int at = y - v * 8;           // the target's place in the vector, if it is there
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo = __uint_as_float(w[i] << 16) * f, hi = __uint_as_float(w[i] & 0xffff0000u) * f;
                if (at == 2 * i) lo = py;
                if (at == 2 * i + 1) hi = py;
                __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
                w[i] = *reinterpret_cast<uint32_t*>(&p);
            }
            e[v] = q[u];
        }
    }
    for (int v = nvec + tid; v < a.lde / 8; v += HEAD_THREADS) e[v] = make_uint4(0u, 0u, 0u, 0u);      // to the end of the last panel
}

// A bucket (slot, then slot -1) sums its tokens' terms, every thread its own tokens in ascending order, then a tree.
struct HeadStats {
    int64_t T;
    int S, cap;
    const int32_t* off;
    const int32_t* slot;
    const float4* terms;
    float* stats;           // or NULL
    int accumulate;
    int32_t* status;
};
__device__ __forceinline__ void head_bucket(const HeadStats& a, int b) {
    __shared__ float4 s_sum[HEAD_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    bool mine = b == a.cap;                 // (tokens that an ill-formed table leaves out count there)
    for (int s = tid; s < a.S; s += HEAD_THREADS) {
        const int t = a.slot[s];
        mine |= t == b;
        if (b == 0) {
            const int x = a.off[s], y = a.off[s + 1];
            if (y < x || x < 0 || y > a.T || (s == 0 && x != 0) || (s == a.S - 1 && y != a.T)) dk_report(a.status, DEV_BAD_TABLE, s);
            if (t < -1 || t >= a.cap) dk_report(a.status, DEV_BAD_INDEX, s);
        }
    }
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (__syncthreads_or(mine)) {
        for (int64_t i = tid; i < a.T; i += HEAD_THREADS) {
            int lo = 0, hi = a.S;           // segments that begin at or before the token: the last of them holds it
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (a.off[mid] <= i) lo = mid + 1; else hi = mid;
            }
            const int t = lo > 0 ? a.slot[lo - 1] : -1;
            if ((t < 0 || t >= a.cap ? a.cap : t) != b) continue;
            const float4 q = a.terms[i];
            v.x += q.x; v.y += q.y; v.z += q.z; v.w += q.w;
        }
    }
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
        v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
        v.w += __shfl_xor_sync(0xffffffffu, v.w, o);
    }
    if (lane == 0) s_sum[warp] = v;
    __syncthreads();
    if (tid < MARLAAS_HEAD_STATS) {
        float x = 0.f;
        for (int w = 0; w < HEAD_THREADS / 32; ++w) x += (&s_sum[w].x)[tid];
        float* out = a.stats + (size_t)b * MARLAAS_HEAD_STATS + tid;
        *out = a.accumulate ? *out + x : x;
    }
}
__global__ void __launch_bounds__(HEAD_THREADS) k_head_stats(const HeadStats a) {
    sm100::dk_wait_prerequisites();
    head_bucket(a, blockIdx.x);
}

// The ranges' partial gradients of a row, summed in their order, scaled and rounded; CTAs behind the rows sum the stats.
__global__ void __launch_bounds__(HEAD_THREADS) k_head_dx(const HeadArgs a, const HeadEpilogue h, int most, int steps, const HeadStats st) {
    sm100::dk_wait_prerequisites();
    if ((int)blockIdx.x >= most) {
        head_bucket(st, (int)blockIdx.x - most);
        return;
    }
    const int rows = min(most, max(0, *h.active - h.row0)), row = blockIdx.x;
    if (row >= rows) return;
    const int nt = (a.d + 255) / 256, tiles = (rows + 255) / 256 * nt, splits = sm100::head_splits(h, tiles, steps, threadIdx.x & 31);
    if (splits == 1) return;
    const float f = h.coef[row];
    bf16* out = a.dx + (int64_t)h.perm[h.row0 + row] * a.lddx;
    for (int v = threadIdx.x; v < a.d / 8; v += HEAD_THREADS) {
        const int c = v * 8;
        const float* in = h.partial + ((size_t)(row >> 8) * nt + (c >> 8)) * 65536 + (size_t)(row & 255) * 256 + (c & 255);
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < splits; ++k) {
            const float4 p = *reinterpret_cast<const float4*>(in), q = *reinterpret_cast<const float4*>(in + 4);
            s[0] += p.x; s[1] += p.y; s[2] += p.z; s[3] += p.w;
            s[4] += q.x; s[5] += q.y; s[6] += q.z; s[7] += q.w;
            in += (size_t)tiles * 65536;
        }
        uint4 o;
        uint32_t* w = &o.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 p = __floats2bfloat162_rn(f * s[2 * i], f * s[2 * i + 1]);
            w[i] = *reinterpret_cast<uint32_t*>(&p);
        }
        *reinterpret_cast<uint4*>(out + c) = o;
    }
}

struct HeadWorkspace {
    int32_t* off;           // [S + 1] host tables
    int32_t* slot;          // [S]
    int32_t* perm;          // [T]
    int32_t* key_off;       // [3]
    int32_t* scratch;
    bf16* rows;             // [T][dp]
    int32_t* row_target;    // [T]
    float* row_coef;        // [T]
    float4* terms;          // [T]
    float2* part;           // [piece][NT]
    float* target_logit;    // [piece]
    bf16* E;                // [piece][lde]
    float* partial;         // [HEAD_ITEMS][256][256]
    int64_t piece, lde, dp, NT;
    size_t total_bytes;
};
static HeadWorkspace carve_head(int64_t T, int64_t d, int64_t V, int32_t S, bool grad, void* base) {
    HeadWorkspace w;
    memset(&w, 0, sizeof(w));
    char* p = (char*)base;
    size_t o = 0;
    auto take = [&](size_t bytes) { char* q = p ? p + o : nullptr; o += align_up(bytes, 256); return q; };
    w.NT = cdiv(V, T <= HEAD_FEW_T ? 128 : 256);
    w.lde = (int64_t)align_up((size_t)V, 64);
    w.dp = (int64_t)align_up((size_t)d, 64);
    // rows of a piece, a multiple of the row tile: by the exponentials' bytes, or without them by the tiles' pairs
    const size_t row_bytes = grad ? (size_t)w.lde * 2 : (size_t)w.NT * 8;
    w.piece = std::min<int64_t>(T, std::max<int64_t>(HEAD_PIECE_BYTES / row_bytes / 256, 1) * 256);
    w.off = (int32_t*)take(sizeof(int32_t) * ((size_t)S + 1));
    w.slot = (int32_t*)take(sizeof(int32_t) * (size_t)S);
    w.perm = (int32_t*)take(sizeof(int32_t) * (size_t)T);
    w.key_off = (int32_t*)take(sizeof(int32_t) * 3);
    w.scratch = (int32_t*)take(sizeof(int32_t) * order_scratch_ints(T, 2));
    w.rows = (bf16*)take(sizeof(bf16) * (size_t)T * (size_t)w.dp);
    w.row_target = (int32_t*)take(sizeof(int32_t) * (size_t)T);
    w.row_coef = (float*)take(sizeof(float) * (size_t)T);
    w.terms = (float4*)take(sizeof(float4) * (size_t)T);
    w.part = (float2*)take(sizeof(float2) * (size_t)w.piece * (size_t)w.NT);
    w.target_logit = (float*)take(sizeof(float) * (size_t)w.piece);
    if (grad) {
        w.E = (bf16*)take(sizeof(bf16) * (size_t)w.piece * (size_t)w.lde);
        const int64_t tiles = cdiv(w.piece, 256) * cdiv(d, 256), steps = cdiv(V, 64) + 1;
        // (one range needs no partial gradients, a range is at least 4 steps, and there are at most 32)
        const int64_t items = std::min<int64_t>(HEAD_ITEMS, tiles * std::min<int64_t>(32, steps / 4));
        w.partial = (float*)take(sizeof(float) * 65536 * (size_t)std::max<int64_t>(items, 0));
    }
    w.total_bytes = o;
    return w;
}

// The bytes of an argument (none, if it is not given).
struct Span {
    const char* name;
    const void* p;
    size_t bytes;
};
static Span matrix_span(const char* name, const void* p, int64_t rows, int64_t ld, int64_t cols) { return {name, p, 2 * (size_t)((rows - 1) * ld + cols)}; }
static bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}

static bool head_sizes_ok(int64_t T, int64_t d, int64_t V) {
    return T >= 0 && T < (1ll << 31) && d >= 8 && d <= MARLAAS_MAX_HEAD_WIDTH && d % 8 == 0 && V >= 1 && V <= MARLAAS_MAX_VOCABULARY;
}

}  // namespace marlaas

using namespace marlaas;

extern "C" {

size_t marlaas_head_cross_entropy_workspace_bytes(const marlaas_pool_t* pool, int64_t T, int64_t d, int64_t V, int32_t num_segments,
                                                  int32_t with_gradient) {
    if (!pool || !head_sizes_ok(T, d, V) || num_segments < 0 || num_segments > MAX_SEGMENTS) return 0;
    return carve_head(T, d, V, num_segments, with_gradient != 0, nullptr).total_bytes;
}

marlaas_status_t marlaas_head_cross_entropy(marlaas_pool_t* pool, int64_t T, int64_t d, int64_t V, const void* x, int64_t ldx,
                                            const void* W, int64_t ldw, const int32_t* targets, const marlaas_segments_t* seg,
                                            const float* weight, float inv_temperature, float grad_scale, void* dx, int64_t lddx,
                                            float* logp, float* stats, void* workspace, size_t workspace_bytes, uint32_t flags,
                                            void* cuda_stream) try {
    const char* fn = "head_cross_entropy";
    if (!pool) return fail(MARLAAS_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (!head_sizes_ok(T, d, V))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: T = %lld, width %lld or V = %lld out of range (a width is a multiple of 8 up to %d, V at most %d)", fn,
                    (long long)T, (long long)d, (long long)V, (int)MARLAAS_MAX_HEAD_WIDTH, (int)MARLAAS_MAX_VOCABULARY);
    if (flags & ~(uint32_t)(MARLAAS_FLAG_HOST_TABLE | MARLAAS_FLAG_VALIDATE_SYNC | MARLAAS_FLAG_ACCUMULATE))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: a flag does not apply to this call", fn);
    if (!(inv_temperature > 0.f) || !std::isfinite(2.f * inv_temperature))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: inv_temperature must be positive, finite and below 1.7e38", fn);
    if (!std::isfinite(grad_scale) || !std::isfinite(grad_scale * inv_temperature))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: grad_scale is not finite", fn);
    // (an output of no tokens may have no address)
    if (T > 0 && !dx && !logp && !stats) return fail(MARLAAS_ERR_INVALID_ARG, "%s: no output", fn);
    if (misaligned(logp, 4) || misaligned(stats, 4) || misaligned(weight, 4))
        return fail(MARLAAS_ERR_INVALID_ARG, "%s: weight, logp or stats is misaligned", fn);
    marlaas_status_t rc;
    if (stats && (rc = check_segments(fn, pool, T, seg, flags, nullptr)) != MARLAAS_OK) return rc;
    const bool accumulate = (flags & MARLAAS_FLAG_ACCUMULATE) != 0, host = stats && (flags & MARLAAS_FLAG_HOST_TABLE) != 0;
    const int32_t S = stats && T > 0 ? seg->num_segments : 0;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    HeadWorkspace ws;
    memset(&ws, 0, sizeof(ws));
    const int32_t *off = stats ? seg->seg_offsets : nullptr, *slot = stats ? seg->seg_slot : nullptr;
    if (T > 0) {
        if ((rc = check_matrix(fn, "x", x, ldx, d)) != MARLAAS_OK) return rc;
        if ((rc = check_matrix(fn, "W", W, ldw, V)) != MARLAAS_OK) return rc;
        if (!targets || misaligned(targets, 4)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: targets is NULL or misaligned", fn);
        if (dx && (rc = check_matrix(fn, "dx", dx, lddx, d)) != MARLAAS_OK) return rc;
        // dx may be x itself: rows are gathered before; other outputs are written while other CTAs still read inputs (of ignored tokens, in the first kernel)
        const bool table = stats && !(flags & MARLAAS_FLAG_HOST_TABLE);
        const Span outs[] = {matrix_span("dx", dx, T, lddx, d), {"logp", logp, 4 * (size_t)T},
                             {"stats", stats, 4 * (size_t)MARLAAS_HEAD_STATS * ((size_t)pool->cap + 1)}};
        const Span ins[] = {matrix_span("x", x, T, ldx, d), matrix_span("W", W, d, ldw, V), {"targets", targets, 4 * (size_t)T},
                            {"weight", weight, 4 * (size_t)T}, {"the segment table", table ? off : nullptr, 4 * ((size_t)S + 1)},
                            {"the segment table", table ? slot : nullptr, 4 * (size_t)S}};
        for (const Span& o : outs)
            for (const Span& i : ins)
                if (overlap(o, i) && !(&o == outs && &i == ins && dx == x && lddx == ldx))
                    return fail(MARLAAS_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, o.name, i.name);
        if (!workspace || misaligned(workspace, 256)) return fail(MARLAAS_ERR_INVALID_ARG, "%s: workspace NULL or misaligned", fn);
        ws = carve_head(T, d, V, S, dx != nullptr, workspace);
        if (workspace_bytes < ws.total_bytes)
            return fail(MARLAAS_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < required %zu", fn, workspace_bytes, ws.total_bytes);
    }
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    if ((rc = reject_host_table_in_capture(fn, flags, st)) != MARLAAS_OK) return rc;
    HeadStats sums;
    memset(&sums, 0, sizeof(sums));
    sums.T = T; sums.S = S; sums.cap = pool->cap; sums.terms = ws.terms; sums.stats = stats; sums.accumulate = accumulate;
    sums.status = pool->d_status;
    if (T > 0) {
        if (host) {     // the copy's source is the call's own and pageable: staged when the copy returns
            std::vector<int32_t> copy((size_t)(ws.slot - ws.off) + (size_t)S);
            std::copy(off, off + S + 1, copy.begin());
            std::copy(slot, slot + S, copy.begin() + (ws.slot - ws.off));
            MARLAAS_CUDA_TRY(cudaMemcpyAsync(ws.off, copy.data(), sizeof(int32_t) * copy.size(), cudaMemcpyHostToDevice, st));
            off = ws.off;
            slot = ws.slot;
        }
        HeadArgs a;
        memset(&a, 0, sizeof(a));
        a.T = T; a.d = (int)d; a.V = (int)V; a.NT = (int)ws.NT; a.tile_shift = T <= HEAD_FEW_T ? 4 : 5; a.dp = (int)ws.dp;
        a.x = (const bf16*)x; a.ldx = ldx; a.targets = targets; a.weight = weight; a.factor = grad_scale * inv_temperature;
        a.perm = ws.perm; a.active = ws.key_off + 1; a.rows = ws.rows; a.row_target = ws.row_target; a.row_coef = ws.row_coef;
        a.E = ws.E; a.lde = ws.lde; a.part = ws.part; a.target_logit = ws.target_logit;
        a.terms = stats ? ws.terms : nullptr; a.logp = logp; a.dx = (bf16*)dx; a.lddx = lddx;
        const unsigned gather = (unsigned)cdiv(T, HEAD_THREADS / 32);
        if (T <= HEAD_SMALL_T) {
            k_head_gather<true><<<gather, HEAD_THREADS, 0, st>>>(a, ws.perm, ws.key_off + 1, pool->d_status);
        } else {
            OrderArgs o;
            memset(&o, 0, sizeof(o));
            o.T = T; o.targets = targets; o.weight = weight; o.V = V; o.nkeys = 2;
            o.perm = ws.perm; o.key_off = ws.key_off;
            if ((rc = launch_order(pool, o, ws.scratch, st)) != MARLAAS_OK) return rc;
            k_head_gather<false><<<gather, HEAD_THREADS, 0, st>>>(a, ws.perm, ws.key_off + 1, pool->d_status);
        }
        MARLAAS_LAUNCH_CHECK("k_head_gather");
        HeadEpilogue h;
        memset(&h, 0, sizeof(h));
        h.active = a.active; h.targets = ws.row_target; h.perm = ws.perm; h.k2 = inv_temperature * HEAD_LOG2E; h.keep = dx != nullptr;
        h.part = ws.part; h.part_ld = (int)ws.NT; h.target_logit = ws.target_logit; h.partial = ws.partial; h.max_items = HEAD_ITEMS;
        h.pairs = head_pairs(pool);
        sums.off = off; sums.slot = slot;
        for (int64_t r0 = 0; r0 < T; r0 += ws.piece) {
            const int64_t rows = std::min<int64_t>(ws.piece, T - r0);
            h.row0 = (int)r0;
            h.coef = ws.row_coef + r0;
            GemmOperands g;
            g.M = rows; g.Nout = V; g.Kc = ws.dp; g.b_cols = d;
            g.A = ws.rows + (size_t)r0 * ws.dp; g.lda = ws.dp;
            g.B = (const bf16*)W; g.ldb = ldw; g.b_mn = true;
            g.C = ws.E; g.ldc = ws.lde;
            g.XA = g.XB = nullptr; g.xa_cols = g.xb_rows = g.xb_ld = 0;
            g.tile_nunits = g.tile_units = nullptr; g.umax = 0;
            rc = T <= HEAD_FEW_T ? launch_head_few(pool, T, d, V, ws.rows, ws.dp, (const bf16*)W, ldw, ws.E, ws.lde, h, st) : launch_head_softmax(pool, g, h, st);
            if (rc != MARLAAS_OK) return rc;
            if (!dx) {
                if ((rc = launch_link("k_head_rows", k_head_rows<false>, dim3((unsigned)rows), HEAD_THREADS, 0, true, st, a, (int)r0)) != MARLAAS_OK) return rc;
                continue;
            }
            if ((rc = launch_link("k_head_rows", k_head_rows<true>, dim3((unsigned)rows), HEAD_THREADS, 0, true, st, a, (int)r0)) != MARLAAS_OK) return rc;
            g.Nout = d; g.Kc = ws.lde; g.b_cols = V;
            g.A = ws.E; g.lda = ws.lde;
            g.b_mn = false;
            g.C = (bf16*)dx; g.ldc = lddx;
            if ((rc = launch_head_grad(pool, g, h, st)) != MARLAAS_OK) return rc;
            const bool with_stats = stats && r0 + rows >= T;
            if ((rc = launch_link("k_head_dx", k_head_dx, dim3((unsigned)(rows + (with_stats ? pool->cap + 1 : 0))), HEAD_THREADS, 0, true, st, a, h, (int)rows,
                                    (int)cdiv(V, 128) * 2, sums)) != MARLAAS_OK) return rc;
        }
    }
    if (stats && (T == 0 || !dx) && (rc = launch_link("k_head_stats", k_head_stats, dim3((unsigned)(pool->cap + 1)), HEAD_THREADS, 0, true, st, sums)) != MARLAAS_OK) return rc;
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "head_cross_entropy: %s", e.what());
}

}  // extern "C"
