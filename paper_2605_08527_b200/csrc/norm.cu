// Layer norm and RMS norm whose gain and bias are each tenant's own, forward and backward (a norm in front of an adapted
// projection; its parameters are trained beside the adapters).  For token i of tenant t, over the d elements of its row:
//     xh = (x - mean) rstd,   rstd = 1 / sqrt(var + eps)          y = xh gain_t + bias_t
//     a = dy gain_t           dx = rstd (a - avg(a) - xh avg(a xh))
//     dgain_t = sum over its tokens of dy xh                      dbias_t = sum of dy
// (RMS norm: mean = 0 and no avg(a).)  Statistics and sums are fp32; x, y, dy, dx are bf16, rounded once when they are written.
// HBM bounds both passes, 4 bytes per element forward and 6 backward, and the issue of instructions nearly as much: unpacking bf16
// and the arithmetic on pairs take 58 % of the issue slots in either pass (16384 x 4096, k_norm_forward 52 us, 5.2 TB/s;
// k_norm_backward 75 us, 5.4 TB/s).  So elements are handled in pairs, sums four at a time, addresses as running pointers, and what
// does not depend on a row (the tenant's parameters, the sums for their gradients) stays where it is from row to row.
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

// Eight elements as four pairs, for the two-element fp32 instructions: both passes are short of issue slots before anything else.
__device__ __forceinline__ void unpack8(const uint4& q, float2 (&f)[4]) {
    const uint32_t* w = &q.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const float2 (&f)[4]) {
    uint4 q;
    uint32_t* w = &q.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 p = __floats2bfloat162_rn(f[i].x, f[i].y);
        w[i] = *reinterpret_cast<uint32_t*>(&p);
    }
    return q;
}
__device__ __forceinline__ void load8(const float* p, float2 (&f)[4]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w);
    f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// ---- both passes ----
// A group of W warps takes a run of rows, B at a time; a thread keeps the same NV x 8 columns throughout, so that its tenant's
// parameters (and the sums for their gradients) stay in registers until the tenant changes: read per row, they were twice the
// bytes of the row itself.  The next batches of rows are on their way as asynchronous copies into shared memory that only the
// copying thread reads, so that the only barriers are those of the rows' sums, of four values at a time.
constexpr int NORM_MAX_GROUPS = 8;
struct GroupSums {
    float v[2][NORM_MAX_GROUPS][4][16];
};

// 16 bytes, or (bytes = 0) as many zeros: what follows needs no branches for ends of rows and batches
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Four sums over a group's threads.  In the warp, lanes hand over half of their values in each of the first two steps: six
// shuffles instead of twenty; eight lanes then hold one value each.  The same tree in every call.
__device__ __forceinline__ void group_sum4(float (&v)[4], GroupSums& s, int& par, int W, int g, int wg, int lane) {
    const bool hi = lane & 16, mid = lane & 8;
    float a0 = hi ? v[2] : v[0], a1 = hi ? v[3] : v[1];
    a0 += __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[2], 16);
    a1 += __shfl_xor_sync(0xffffffffu, hi ? v[1] : v[3], 16);
    float x = (mid ? a1 : a0) + __shfl_xor_sync(0xffffffffu, mid ? a0 : a1, 8);
    x += __shfl_xor_sync(0xffffffffu, x, 4);
    x += __shfl_xor_sync(0xffffffffu, x, 2);
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    const int k = lane >> 3;                    // the value that this lane holds
    if (W > 1) {
        if ((lane & 7) == 0) s.v[par][g][k][wg] = x;
        asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "r"(32 * W) : "memory");
        const float* part = s.v[par][g][k] + (lane & 7);
        x = (lane & 7) < W ? part[0] : 0.f;
        if (W > 8) x += (lane & 7) + 8 < W ? part[8] : 0.f;
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        par ^= 1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(0xffffffffu, x, 8 * i);
}

// The segment of token i, a.S for a token that an ill-formed table leaves out.  A warp looks together, 32 places at a time: a table
// of 1024 segments is two loads in a row.
__device__ __forceinline__ int segment_of(const NormArgs& a, int i, int lane) {
    int lo = 0, hi = a.S;                       // the segments before lo end at or before i; that of hi, if there is one, behind it
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, m = lo + lane * step;
        const unsigned behind = __ballot_sync(0xffffffffu, m >= hi || a.off[m + 1] > i);
        const int before = behind ? __ffs(behind) - 1 : 32;
        hi = min(hi, lo + before * step);
        if (before > 0) lo += (before - 1) * step + 1;
    }
    return lo;
}
__device__ __forceinline__ int norm_slot(const NormArgs& a, int seg) {
    const int t = seg < a.S ? a.slot[seg] : -1;
    return t < 0 || t >= a.cap ? a.cap : t;
}
__device__ __forceinline__ void check_table(const NormArgs& a) {
    for (int64_t s = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; s < a.S; s += (int64_t)gridDim.x * blockDim.x) {
        const int p = a.off[s], q = a.off[s + 1], t = a.slot[s];
        if (q < p || p < 0 || q > a.T || (s == 0 && p != 0) || (s == a.S - 1 && q != a.T)) dk_report(a.status, DEV_BAD_TABLE, (int)s);
        if (t < -1 || t >= a.cap) dk_report(a.status, DEV_BAD_INDEX, (int)s);
    }
}

// ---- forward ----
template <int NV, int B, int STAGES, int THREADS, int PER_SM, bool RMS>
__global__ void __launch_bounds__(THREADS, PER_SM) k_norm_forward(const NormArgs a, int W, int G) {
    extern __shared__ uint4 s_ring[];           // [STAGES][B][NV][THREADS]
    __shared__ GroupSums s_sums;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = warp / W, wg = warp % W, l = wg * 32 + lane;
    const int nvec = a.d / 8;
    const float inv_d = 1.f / (float)a.d;
    check_table(a);
    const int64_t first = ((int64_t)blockIdx.x * G + g) * a.rows_per_group;
    if (first >= a.T) return;                   // (a group synchronises with itself alone)
    const int n = (int)min(a.rows_per_group, a.T - first);      // rows of the group
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + threadIdx.x * 16;
    bool mine[NV];
    uint32_t bytes[NV], at[NV];                 // what a lane copies of a vector's 16 bytes, and from where in the row
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = l + j * 32 * W;
        mine[j] = c < nvec;
        bytes[j] = mine[j] ? 16 : 0;
        at[j] = mine[j] ? (uint32_t)c * 16 : 0;
    }
    // the next row that is fetched; behind the group's last row it is read again, and dropped
    const char* px = reinterpret_cast<const char*>(a.x + first * a.ldx);
    char* py = reinterpret_cast<char*>(a.y + first * a.ldy);
    const int64_t step_x = a.ldx * 2, step_y = a.ldy * 2;
    int left = n - 1;                           // rows behind px
    auto fetch = [&](int st) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
#pragma unroll
            for (int j = 0; j < NV; ++j) copy16(ring + (uint32_t)(((st * B + b) * NV + j) * THREADS * 16), px + at[j], bytes[j]);
            if (left-- > 0) px += step_x;
        }
        copy_commit();
    };
    auto element = [&](int st, int b, int j) { return s_ring[((st * B + b) * NV + j) * THREADS + threadIdx.x]; };
#pragma unroll
    for (int u = 0; u < STAGES - 1; ++u) fetch(u);
    int par = 0, st = 0, seg = -1, seg_end = 0; // seg_end: the group's first row of a later segment
    float2 gain[NV][4], bias[NV][4], f[4];
    auto next_tenant = [&](int r) {             // the segment of the group's row r: the next one, or else looked for; its parameters
        const int i = (int)first + r;
        int lo = seg + 1;
        if (seg < 0 || lo >= a.S || a.off[lo] > i || a.off[lo + 1] <= i) lo = segment_of(a, i, lane);
        seg_end = r + 1;
        if (lo < a.S) {
            seg = lo;
            seg_end = (int)min((int64_t)n, (int64_t)a.off[lo + 1] - first);
        }
        const int t = norm_slot(a, lo);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const size_t c = (size_t)t * a.d + at[j] / 2;
            load8(a.gain + c, gain[j]);
            if (a.bias) load8(a.bias + c, bias[j]);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) bias[j][e] = make_float2(0.f, 0.f);
        }
    };
    next_tenant(0);                             // (while the first rows are on their way)
    for (int r = 0; r < n; r += B) {
        fetch(st == 0 ? STAGES - 1 : st - 1);
        copy_wait<STAGES - 1>();
        float v[4] = {0.f, 0.f, 0.f, 0.f}, mean[4] = {0.f, 0.f, 0.f, 0.f};
        if (!RMS) {
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    unpack8(element(st, b, j), f);
                    const float2 s = __fadd2_rn(__fadd2_rn(f[0], f[1]), __fadd2_rn(f[2], f[3]));
                    v[b] += s.x + s.y;
                }
            group_sum4(v, s_sums, par, W, g, wg, lane);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                // (divided: the sum of a constant row is exact, and its quotient the constant; times 1 / d it may miss by an ulp)
                mean[b] = __fdiv_rn(v[b], (float)a.d);
                v[b] = 0.f;
            }
        }
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                unpack8(element(st, b, j), f);
                float2 s = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 c = RMS ? f[e] : __fadd2_rn(f[e], both(-mean[b]));
                    s = __ffma2_rn(c, c, s);
                }
                v[b] += RMS || mine[j] ? s.x + s.y : 0.f;
            }
        group_sum4(v, s_sums, par, W, g, wg, lane);
#pragma unroll
        for (int b = 0; b < B; ++b) {
            v[b] = rsqrtf(fmaf(v[b], inv_d, a.eps));
            if (r + b < n) {
                if (r + b >= seg_end) next_tenant(r + b);
                const float2 scale = both(v[b]), shift = both(-mean[b]);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    unpack8(element(st, b, j), f);
#pragma unroll
                    for (int e = 0; e < 4; ++e)         // (x - mean, so that a constant row is its bias)
                        f[e] = __ffma2_rn(__fmul2_rn(RMS ? f[e] : __fadd2_rn(f[e], shift), scale), gain[j][e], bias[j][e]);
                    if (mine[j]) *reinterpret_cast<uint4*>(py + at[j]) = pack8(f);
                }
                py += step_y;
            }
        }
        if (l == 0) {
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (r + b < n) {
                    if (a.mean) a.mean[first + r + b] = mean[b];
                    if (a.rstd) a.rstd[first + r + b] = v[b];
                }
        }
        st = st == STAGES - 1 ? 0 : st + 1;
    }
}

// ---- backward ----
// The rows are taken in the order of their tenants.  The sums of a (group, tenant) pair go to partial[group + tenant]: both only
// rise along the ordered tokens, so no two pairs share a place, and the order of all additions depends on the sizes and the
// table alone.  A batch of few segments is taken as it comes (perm = NULL), without the launches that order it: the sums of a
// (group, segment) pair go to partial[group + segment], for the same reason.
template <int NV, int B, int STAGES, int THREADS, int PER_SM, bool RMS>
__global__ void __launch_bounds__(THREADS, PER_SM) k_norm_backward(const NormArgs a, int W, int G) {
    // four vectors per lane leave no registers for the gains: each thread keeps its own behind the ring
    constexpr bool GAIN_SHARED = NV == 4;
    extern __shared__ uint4 s_ring[];           // [STAGES][B][x, dy][NV][THREADS]
    float4* const s_gain = reinterpret_cast<float4*>(s_ring + STAGES * B * 2 * NV * THREADS) + threadIdx.x;     // [NV][2][THREADS]
    __shared__ GroupSums s_sums;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = warp / W, wg = warp % W, l = wg * 32 + lane;
    const int nvec = a.d / 8;
    const float inv_d = 1.f / (float)a.d;
    const int64_t q = (int64_t)blockIdx.x * G + g, first = q * a.rows_per_group;
    sm100::dk_wait_prerequisites();
    sm100::dk_launch_dependents();
    const bool ordered = a.perm != nullptr;
    if (!ordered) check_table(a);
    if (first >= a.T) return;
    const int n = (int)min(a.rows_per_group, a.T - first);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + threadIdx.x * 16;
    bool mine[NV];
    uint32_t at[NV];                            // a lane's bytes of a row
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = l + j * 32 * W;
        mine[j] = c < nvec;
        at[j] = mine[j] ? (uint32_t)c * 16 : 0;
    }
    const char* const px = reinterpret_cast<const char*>(a.x);
    const char* const pdy = reinterpret_cast<const char*>(a.dy);
    char* const py = reinterpret_cast<char*>(a.y);
    const int64_t step_x = a.ldx * 2, step_dy = a.lddy * 2, step_y = a.ldy * 2;
    auto fetch = [&](const int (&tok)[B], int r, int st) {      // (rows past the end are zeros)
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const char* x = px + tok[b] * step_x;
            const char* dy = pdy + tok[b] * step_dy;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t to = ring + (uint32_t)((((st * B + b) * 2) * NV + j) * THREADS * 16), bytes = r + b < n && mine[j] ? 16 : 0;
                copy16(to, x + at[j], bytes);
                copy16(to + (uint32_t)(NV * THREADS * 16), dy + at[j], bytes);
            }
        }
        copy_commit();
    };
    auto element = [&](int st, int b, int which, int j) { return s_ring[(((st * B + b) * 2 + which) * NV + j) * THREADS + threadIdx.x]; };
    // tok[u]: the tokens of the batch u steps ahead; behind the group's last row, that row's
    int tok[STAGES][B];
    auto tokens = [&](int (&t)[B], int r) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
            t[b] = (int)first + min(r + b, n - 1);
            if (ordered) t[b] = a.perm[t[b]];
        }
    };
#pragma unroll
    for (int u = 0; u < STAGES; ++u) tokens(tok[u], u * B);
    // the moments of the next batch are asked for a batch ahead, too
    float mean_next[B], rstd_next[B];
    auto moments = [&](const int (&t)[B]) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
            mean_next[b] = RMS ? 0.f : a.mean_in[t[b]];
            rstd_next[b] = a.rstd_in[t[b]];
        }
    };
    moments(tok[0]);
#pragma unroll
    for (int u = 0; u < STAGES - 1; ++u) fetch(tok[u], u * B, u);
    int key = -1, par = 0, st = 0, key_end = 0;     // the tenant, or the segment; key_end: the group's first row of a later one
    float2 gain_kept[GAIN_SHARED ? 1 : NV][4], sg[NV][4], sb[NV][4];
    auto flush = [&]() {
        float* out = a.partial + (size_t)(q + key) * 2 * a.d;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = l + j * 32 * W;
            if (mine[j]) {
                float4* o = reinterpret_cast<float4*>(out + v * 8);
                o[0] = make_float4(sg[j][0].x, sg[j][0].y, sg[j][1].x, sg[j][1].y);
                o[1] = make_float4(sg[j][2].x, sg[j][2].y, sg[j][3].x, sg[j][3].y);
                if (a.dbias) {
                    o = reinterpret_cast<float4*>(out + a.d + v * 8);
                    o[0] = make_float4(sb[j][0].x, sb[j][0].y, sb[j][1].x, sb[j][1].y);
                    o[1] = make_float4(sb[j][2].x, sb[j][2].y, sb[j][3].x, sb[j][3].y);
                }
            }
        }
    };
    auto load_gain = [&](int k) {
        const int t = ordered ? k : norm_slot(a, k);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float2 w[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
            if (mine[j]) load8(a.gain + (size_t)t * a.d + at[j] / 2, w);
            if (GAIN_SHARED) {
                s_gain[2 * j * THREADS] = make_float4(w[0].x, w[0].y, w[1].x, w[1].y);
                s_gain[(2 * j + 1) * THREADS] = make_float4(w[2].x, w[2].y, w[3].x, w[3].y);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) gain_kept[j][e] = w[e];
            }
        }
    };
    auto gains = [&](int j, float2 (&w)[4]) {
        if (GAIN_SHARED) {
            const float4 p = s_gain[2 * j * THREADS], q = s_gain[(2 * j + 1) * THREADS];
            w[0] = make_float2(p.x, p.y); w[1] = make_float2(p.z, p.w);
            w[2] = make_float2(q.x, q.y); w[3] = make_float2(q.z, q.w);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = gain_kept[j][e];
        }
    };
    auto next_tenant = [&](int r) {             // the next tenant that has tokens; its gain, and sums of 0
        if (ordered) {
            do key_end = (int)min((int64_t)n, a.key_off[++key + 1] - first); while (key_end <= r);
        } else {
            // (tokens that an ill-formed table leaves out are a segment behind the last one)
            key = segment_of(a, (int)first + r, lane);
            key_end = key < a.S ? (int)min((int64_t)n, a.off[key + 1] - first) : n;
        }
        load_gain(key);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sg[j][e] = sb[j][e] = make_float2(0.f, 0.f);
        }
    };
    for (int r = 0; r < n; r += B) {
        fetch(tok[STAGES - 1], r + (STAGES - 1) * B, st == 0 ? STAGES - 1 : st - 1);
        float mean[B], rstd[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            mean[b] = mean_next[b];
            rstd[b] = rstd_next[b];
        }
        moments(tok[1]);
        if (r >= key_end) {
            if (key >= 0 && a.partial) flush();
            next_tenant(r);
        }
        const int key0 = key;                   // (the batch's second row may be the next one's)
        copy_wait<STAGES - 1>();
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        float2 x[4], dy[4], gain[4];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (b == 1 && r + 1 >= key_end && r + 1 < n) {
                if (a.partial) flush();
                next_tenant(r + 1);
            }
            float2 s = make_float2(0.f, 0.f), u = s;
#pragma unroll
            for (int j = 0; j < NV; ++j) {      // (dy is zero past the row's and the batch's end and adds nothing)
                unpack8(element(st, b, 0, j), x);
                unpack8(element(st, b, 1, j), dy);
                gains(j, gain);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (x - mean, so that a sum of one token keeps its digits where x is near the mean)
                    const float2 xh = __fmul2_rn(RMS ? x[e] : __fadd2_rn(x[e], both(-mean[b])), both(rstd[b]));
                    const float2 av = __fmul2_rn(dy[e], gain[e]);
                    sg[j][e] = __ffma2_rn(dy[e], xh, sg[j][e]);
                    sb[j][e] = __fadd2_rn(dy[e], sb[j][e]);
                    if (!RMS) s = __fadd2_rn(av, s);
                    u = __ffma2_rn(av, xh, u);
                }
            }
            v[2 * b] = s.x + s.y;
            v[2 * b + 1] = u.x + u.y;
        }
        if (a.y) {
            group_sum4(v, s_sums, par, W, g, wg, lane);
#pragma unroll
            for (int b = B - 1; b >= 0; --b) {
                if (r + b < n) {
                    // dx = a rstd + (x - mean) k + c
                    const float mx = v[2 * b + 1] * inv_d, k = -rstd[b] * rstd[b] * mx, c = -rstd[b] * (v[2 * b] * inv_d);
                    char* const to = py + tok[0][b] * step_y;
                    if (b == 0 && key0 != key) load_gain(key0);
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        unpack8(element(st, b, 0, j), x);
                        unpack8(element(st, b, 1, j), dy);
                        gains(j, gain);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[e] = __ffma2_rn(__fmul2_rn(dy[e], gain[e]), both(rstd[b]), RMS ? __fmul2_rn(x[e], both(k)) : __ffma2_rn(__fadd2_rn(x[e], both(-mean[b])), both(k), both(c)));
                        if (mine[j]) *reinterpret_cast<uint4*>(to + at[j]) = pack8(x);
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < STAGES - 1; ++u)
#pragma unroll
            for (int b = 0; b < B; ++b) tok[u][b] = tok[u + 1][b];
        tokens(tok[STAGES - 1], r + STAGES * B);
        st = st == STAGES - 1 ? 0 : st + 1;
        if (a.y && key0 != key) load_gain(key);
    }
    if (a.partial) flush();
}

// dgain and dbias of one tenant, 128 columns per CTA, four per lane: the warps share the tenant's partial sums, then add up in their
// order.
__global__ void __launch_bounds__(1024) k_norm_reduce(const NormArgs a) {
    extern __shared__ float4 s_sum[];           // [2][warps][32], then a range per thread
    __shared__ int s_warp[32];
    int2* const s_range = reinterpret_cast<int2*>(s_sum + 2 * blockDim.x);
    const int key = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5, c = blockIdx.x * 128 + lane * 4;
    const int rows = (int)a.rows_per_group;
    float4 g = make_float4(0.f, 0.f, 0.f, 0.f), h = g;
    int seen = 0;                               // places before the present range
    auto add = [&](int from, int to) {
        if (c < a.d) {
#pragma unroll 4
            for (int q = from + (warp + seen) % warps; q < to; q += warps) {
                const float* in = a.partial + (size_t)q * 2 * a.d + c;
                const float4 x = *reinterpret_cast<const float4*>(in);
                g.x += x.x; g.y += x.y; g.z += x.z; g.w += x.w;
                if (a.dbias) {
                    const float4 y = *reinterpret_cast<const float4*>(in + a.d);
                    h.x += y.x; h.y += y.y; h.z += y.z; h.w += y.w;
                }
            }
        }
        seen += to - from;
    };
    if (a.perm) {
        sm100::dk_wait_prerequisites();
        const int b = a.key_off[key], e = a.key_off[key + 1];
        if (e > b) add(b / rows + key, (e - 1) / rows + key + 1);
    } else {
        // the tenant's segments, and what lies behind the last one
        for (int s0 = 0; s0 <= a.S; s0 += blockDim.x) {
            const int s = s0 + tid;
            int b = 0, e = 0;
            if (s <= a.S && norm_slot(a, s) == key) {
                b = s == 0 ? 0 : max(0, a.off[s]);
                e = s < a.S ? min((int)a.T, a.off[s + 1]) : (int)a.T;
            }
            const unsigned bal = __ballot_sync(0xffffffffu, e > b);
            if (lane == 0) s_warp[warp] = __popc(bal);
            __syncthreads();
            int at = __popc(bal & ((1u << lane) - 1u)), n = 0;
            for (int w = 0; w < warps; ++w) {
                at += w < warp ? s_warp[w] : 0;
                n += s_warp[w];
            }
            if (e > b) s_range[at] = make_int2(b / rows + s, (e - 1) / rows + s + 1);
            __syncthreads();
            sm100::dk_wait_prerequisites();
            for (int k = 0; k < n; ++k) add(s_range[k].x, s_range[k].y);
        }
    }
    if (seen > 0) {
        s_sum[tid] = g;
        s_sum[blockDim.x + tid] = h;
        __syncthreads();
    }
    if (warp >= 2 || c >= a.d) return;
    float* out = warp == 0 ? a.dgain : a.dbias;
    if (!out) return;
    float4* dst = reinterpret_cast<float4*>(out + (size_t)key * a.d + c);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (seen > 0)
        for (int w = 0; w < warps; ++w) {
            const float4 x = s_sum[(warp * warps + w) * 32 + lane];
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
    if (a.accumulate) {
        const float4 x = *dst;
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    *dst = v;
}

// How a pass cuts a batch: vectors per lane, warps per row and rows of a CTA at a time, groups in all and their rows.
// As many vectors per lane as registers allow: half of a row's instructions do not depend on how many elements a lane has.
// Backward 16384 x 5120: four per lane 92 us, two 105; 2000 x 16384: 54 us, with two (and 1024 threads, whose registers spill) 114;
// below 2048 elements four leave too few warps per row's sum or idle lanes (2048: 41 us against 40).
struct NormPlan {
    int NV, W, G;
    int64_t groups, rows;
};
static NormPlan norm_plan(const marlaas_pool* pool, int64_t T, int d, bool backward) {
    NormPlan p;
    const int nvec = d / 8;
    p.NV = nvec >= 256 ? 4 : nvec >= 64 ? 2 : 1;
    p.W = (int)cdiv(nvec, 32 * p.NV);
    p.G = (int)std::max<int64_t>(1, std::min<int64_t>({NORM_MAX_GROUPS, (p.NV == 4 ? 16 : 8) / p.W, cdiv(T, pool->sm_count)}));
    const int threads = 32 * p.W * p.G;
    const int64_t most = (int64_t)pool->sm_count * std::max(1, (p.NV == 4 || (backward && p.NV == 2) ? 512 : 768) / threads) * p.G;
    // (a group's partial sums cost as much as four of its rows: backward, no group takes fewer)
    p.rows = std::max<int64_t>(cdiv(T, most), backward ? 4 : 1);
    p.groups = cdiv(cdiv(T, p.rows), p.G) * p.G;
    return p;
}

// Whether backward takes a batch as it comes.  Each segment then costs sums of its own, 8 bytes per column to write and to read
// again, where the order costs three launches in a row, about 12 us or 60 MB (8000 x 1600 in 62 segments: 34 us as it comes, 41 ordered).
static bool norm_as_it_comes(int64_t d, int32_t S) { return S <= 8192 && 16 * d * S <= 60000000; }

struct NormWorkspace {
    int32_t* off;           // [S + 1] host tables
    int32_t* slot;          // [S]
    int32_t* perm;          // [T]; these three for batches that are ordered
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
        const NormPlan n = norm_plan(pool, T, (int)d, true);
        const bool ordered = !norm_as_it_comes(d, S);
        if (ordered) {
            w.perm = (int32_t*)take(sizeof(int32_t) * (size_t)T);
            w.key_off = (int32_t*)take(sizeof(int32_t) * ((size_t)pool->cap + 2));
            w.scratch = (int32_t*)take(sizeof(int32_t) * order_scratch_ints(T, pool->cap + 1));
        }
        w.partial = (float*)take(sizeof(float) * (size_t)(n.groups + (ordered ? pool->cap : S) + 1) * 2 * (size_t)d);
    }
    w.total_bytes = o;
    return w;
}

// Instances by the vectors per lane.  CTAs share an SM so that no instance spills: what is left of L1 beside the rows on their way
// does not hold spilled registers (backward 16384 x 4096 with 80 registers per thread, RMS: 183 us, with 114 and two CTAs instead
// of three: 74).
template <int NV, int THREADS, int PER_SM, bool RMS>
static marlaas_status_t launch_norm_t(const marlaas_pool* pool, const NormArgs& a, const NormPlan& n, bool backward, cudaStream_t st) {
    constexpr int STAGES = NV == 1 ? 3 : 2, FB = NV == 4 ? 2 : 4, BB = NV == 4 ? 1 : 2;
    const int threads = 32 * n.W * n.G;
    const size_t fwd = (size_t)STAGES * FB * NV * 16, bwd = (size_t)STAGES * BB * 2 * NV * 16 + (NV == 4 ? NV * 32 : 0);      // shared bytes per thread
    auto* kf = k_norm_forward<NV, FB, STAGES, THREADS, PER_SM, RMS>;
    auto* kb = k_norm_backward<NV, BB, STAGES, THREADS, NV == 2 && PER_SM == 3 ? 2 : PER_SM, RMS>;
    static bool attr_set[64] = {};
    if (pool->device >= 64 || !attr_set[pool->device]) {
        MARLAAS_CUDA_TRY(cudaFuncSetAttribute(kf, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)std::min<size_t>(fwd * THREADS, 200 * 1024)));
        MARLAAS_CUDA_TRY(cudaFuncSetAttribute(kb, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)std::min<size_t>(bwd * THREADS, 200 * 1024)));
        if (pool->device < 64) attr_set[pool->device] = true;
    }
    // (backward: behind the order's kernels, if there are any)
    return launch_link(backward ? "k_norm_backward" : "k_norm_forward", backward ? kb : kf, dim3((unsigned)(n.groups / n.G)), (unsigned)threads,
                       (backward ? bwd : fwd) * THREADS, a.perm != nullptr, st, a, n.W, n.G);
}
static marlaas_status_t launch_norm(const marlaas_pool* pool, NormArgs a, bool rms, bool backward, cudaStream_t st) {
    const NormPlan n = norm_plan(pool, a.T, a.d, backward);
    a.rows_per_group = n.rows;
#define NORM_GO(nv, threads, per) (rms ? launch_norm_t<nv, threads, per, true>(pool, a, n, backward, st) : launch_norm_t<nv, threads, per, false>(pool, a, n, backward, st))
    if (n.NV == 1) return NORM_GO(1, 256, 3);
    return n.NV == 2 ? NORM_GO(2, 256, 3) : NORM_GO(4, 512, 1);
#undef NORM_GO
}

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
    if ((rc = launch_norm(pool, a, (flags & MARLAAS_FLAG_RMS_NORM) != 0, false, st)) != MARLAAS_OK) return rc;
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
    // (a dx of no tokens may have no address)
    if (T > 0 && !dx && !dgain && !dbias) return fail(MARLAAS_ERR_INVALID_ARG, "%s: no output", fn);
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
    const NormPlan n = norm_plan(pool, T, (int)d, true);
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
    if (a.perm) {
        OrderArgs o;
        memset(&o, 0, sizeof(o));
        o.T = T; o.S = a.S; o.off = a.off; o.slot = a.slot; o.cap = pool->cap; o.nkeys = pool->cap + 1;
        o.perm = ws.perm; o.key_off = ws.key_off;
        if ((rc = launch_order(pool, o, ws.scratch, st)) != MARLAAS_OK) return rc;
    }
    rc = launch_norm(pool, a, rms, true, st);
    if (rc != MARLAAS_OK) return rc;
    if (a.partial) {
        // as many warps as let all CTAs run at once
        const int64_t ctas = cdiv(d, 128) * (pool->cap + 1);
        int warps = 8;
        while (warps < 32 && warps * 32 < n.groups && ctas * warps * 2 <= (int64_t)pool->sm_count * 64) warps *= 2;
        rc = launch_link("k_norm_reduce", k_norm_reduce, dim3((unsigned)cdiv(d, 128), (unsigned)(pool->cap + 1)), (unsigned)(warps * 32),
                         (size_t)warps * 32 * (2 * sizeof(float4) + sizeof(int2)), true, st, a);
        if (rc != MARLAAS_OK) return rc;
    }
    return finish(pool, flags, st);
} catch (const std::exception& e) {
    return fail(MARLAAS_ERR_INVALID_ARG, "layer_norm_backward: %s", e.what());
}

}  // extern "C"
