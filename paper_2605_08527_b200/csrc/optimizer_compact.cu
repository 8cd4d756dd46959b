// AdamW and commit with both moments in 8 bits (Algorithm 1: "PolicyUpdate" and the commit of the new adapter version;
// Methods, Multi-Task Manager: per-task optimizer state, which at 8 bytes per element is four times the bf16 adapter
// itself).  The state's format is in marlaas.h.  Per element: gradient 4 B read, master 4 + 4, moments 2.06 + 2.06, the
// pool's bf16 2 written = 18.1 bytes and no reuse: bound by HBM, with the arithmetic not far behind (90 instructions per
// element, most of them integer work on codes and random bits: the ALU pipes are two thirds busy at the rate reached).
// Measured: 87 us for 32 tenants of rank 32 over a 4096 x (3 x 4096) pool (25.2 M elements, 456 MB, 0.81 of the copy rate;
// 155 us with one element at a time and IEEE division and root), 113 us for rank 128 over 4096 x 4096 (0.83), 39.1 us for ranks
// 8 to 64 over 5120 x 5120 (9.8 M elements, 0.71: 2.7 rounds of units over the places for CTAs).
#include <string.h>

#include <cmath>

#include "internal.cuh"

namespace marlaas {

constexpr int OC_THREADS = 256;
constexpr int OC_BLOCK = 256;               // elements that share their exponents: one warp, 8 per lane
constexpr int OC_STATE_BYTES = 528;
constexpr int OC_UNIT = 2048;               // elements of B (and at least, of A) per CTA, or OC_LONG times as many
constexpr int OC_LONG = 4;
constexpr int OC_MAX_TENANTS = 256;         // tenants per launch
constexpr uint32_t OC_M_ORDERS = 15, OC_V_ORDERS = 31;      // binary orders below the block's largest exponent

struct CompactTenant {
    const float* dA;
    const float* dB;
    float* A;
    float* B;
    uint8_t* sA;
    uint8_t* sB;
    int32_t slot;
    uint16_t rank, vec;     // vec: gradients and masters are 16-byte aligned
    uint32_t key[2 * MARLAAS_MAX_PARTS];    // of the random bits: A and B of each projection
};
struct CompactHyper {
    float b1, b2, one_b1, one_b2, gscale;
    float sqrt_c2, eps, lr_c1, lr_wd;       // c1 = 1 / (1 - beta1^step), c2 = 1 / (1 - beta2^step)
};
// The table of a launch; three sizes, so that a few tenants do not pay for the parameters of 256.
template <int N>
struct CompactArgs {
    int n, P, RP, cap;
    int64_t K, ldB;
    int64_t part_begin[MARLAAS_MAX_PARTS + 1];
    CompactHyper h;
    int unit;                       // elements of B per CTA
    bf16* At;
    bf16* Bs;
    int32_t first[2 * N + 1];       // first CTA of tenant t's A (2t) and B (2t + 1)
    CompactTenant t[N];
};

// Random bits of an element: two rounds of xor-shift and multiplication by odd constants (2^32 divided by the golden ratio,
// and by the square root of 2), a bijection of the 32-bit numbers.
__host__ __device__ __forceinline__ uint32_t mix32_open(uint32_t x) {      // without the last step
    x = (x ^ (x >> 16)) * 0x9E3779B9u;
    return (x ^ (x >> 15)) * 0xB504F333u;
}
static uint32_t mix32(uint32_t x) {
    x = mix32_open(x);
    return x ^ (x >> 16);
}
static uint32_t stream_key(uint64_t seed, uint64_t step, uint64_t tenant, uint32_t matrix) {
    const uint32_t w[7] = {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32),
                           (uint32_t)tenant, (uint32_t)(tenant >> 32), matrix};
    uint32_t k = 0;
    for (int i = 0; i < 7; ++i) k = mix32((k + 0x9E3779B9u) ^ w[i]);
    return k;
}

// Codes count in steps of 2^20 of the fp32 bit pattern (sign cut off): exponent and 3 mantissa bits.
__device__ __forceinline__ uint32_t code_base(uint32_t E, uint32_t orders) { return E > orders ? (E - orders) * 8 : 0; }
__device__ __forceinline__ float code_value(uint32_t c, uint32_t base20) { return c ? __uint_as_float((c << 20) + base20) : 0.f; }
__device__ __forceinline__ uint32_t byte_of(uint32_t w, int i) { return __byte_perm(w, 0, 0x4440 + i); }
// Byte i of w in bits 16 to 23, so that one multiply-add by 16 makes a code's bit pattern of it.
__device__ __forceinline__ uint32_t byte_at_16(uint32_t w, int i) { return __byte_perm(w, 0, 0x4044 + (i << 8)); }
// Four numbers as unsigned bytes, cut off at 0 and 255.
__device__ __forceinline__ uint32_t bytes(int32_t a, int32_t b, int32_t c, int32_t d) {
    uint32_t r;
    asm("{\n\t.reg .b32 t;\n\t"
        "cvt.pack.sat.u8.s32.b32 t, %4, %3, 0;\n\t"
        "cvt.pack.sat.u8.s32.b32 %0, %2, %1, t;\n\t}"
        : "=r"(r) : "r"(a), "r"(b), "r"(c), "r"(d));
    return r;
}
// The top bits of four words as 0x80 in four bytes.
__device__ __forceinline__ uint32_t signs(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410) & 0x80808080u;
}
// The magnitude to store where a block holds numbers that are too large: not finite -> 0; never so large that rounding up
// leaves the finite numbers.
constexpr uint32_t OC_LARGEST = 0x7f700000u;
__device__ __forceinline__ uint32_t magnitude(uint32_t b) { return b >= 0x7f800000u ? 0u : min(b, OC_LARGEST); }
// The exponent that holds a block's largest magnitude also after rounding up.
__device__ __forceinline__ uint32_t block_exponent(uint32_t largest) { return (largest + 0xfffffu) >> 23; }
// (below the block's range: 0 or negative)
__device__ __forceinline__ int32_t code_of(uint32_t mag, uint32_t rnd16, uint32_t base20) { return (int32_t)(rnd16 * 16u + mag - base20) >> 20; }
__device__ __forceinline__ float sqrt_approx(float x) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Products and sums of two numbers, each rounded by itself.  (Two-element instructions are no use here: a product and the sum
// that takes it become one multiply-add, also with their rounding written out, and that moves about one code in a million.)
__device__ __forceinline__ float2 mul_rn(float2 a, float2 b) { return make_float2(__fmul_rn(a.x, b.x), __fmul_rn(a.y, b.y)); }
__device__ __forceinline__ float2 add_rn(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }

// What a lane holds of a block of 256 elements: elements 4 lane .. 4 lane + 3 and 128 further on.
struct CompactLane {
    float4 g[2], th[2];
    uint32_t m[2], v[2], E;
};
// `left`: elements of the matrix from the block's first on (a multiple of 8); below 256 the rest of the block is zeros.
__device__ __forceinline__ void compact_load(CompactLane& x, const float* __restrict__ grad, const float* __restrict__ theta,
                                             const uint8_t* __restrict__ blk, int left, bool vec, int lane) {
    if (left >= OC_BLOCK && vec) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            x.m[q] = reinterpret_cast<const uint32_t*>(blk)[32 * q + lane];
            x.v[q] = reinterpret_cast<const uint32_t*>(blk + 256)[32 * q + lane];
            x.g[q] = __ldcs(reinterpret_cast<const float4*>(grad) + 32 * q + lane);
            x.th[q] = __ldcs(reinterpret_cast<const float4*>(theta) + 32 * q + lane);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = 128 * q + 4 * lane;
            x.m[q] = x.v[q] = 0;
            x.g[q] = x.th[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (e < left) {
                x.m[q] = reinterpret_cast<const uint32_t*>(blk)[32 * q + lane];
                x.v[q] = reinterpret_cast<const uint32_t*>(blk + 256)[32 * q + lane];
                x.g[q] = make_float4(grad[e], grad[e + 1], grad[e + 2], grad[e + 3]);
                x.th[q] = make_float4(theta[e], theta[e + 1], theta[e + 2], theta[e + 3]);
            }
        }
    }
    x.E = *reinterpret_cast<const uint16_t*>(blk + 512);
}

// The step of a block: writes masters and state, leaves the new masters in x.th.  `rnd`: the block's first element + key.
__device__ __forceinline__ void compact_step(CompactLane& x, const CompactHyper& h, float* __restrict__ theta, uint8_t* __restrict__ blk,
                                             int left, bool vec, uint32_t rnd, int lane) {
    const uint32_t bm = code_base(x.E & 255u, OC_M_ORDERS) << 20, bv = code_base(x.E >> 8, OC_V_ORDERS) << 20;
    uint32_t mb[8], vb[8], top_m = 0, top_v = 0;
    // A v of 0 in a block that holds an m of 1 or more: the square of an earlier gradient left fp32's range (a positive v never
    // becomes 0, and where a square was too small for fp32 the m is below 2^-50, a code of 0 in such a block).  That m over the
    // root of an ordinary v would throw the master many orders of magnitude; both start anew from 0.  (Masks, not a branch for
    // such blocks: 32 tenants of rank 32 over 4096 x (3 x 4096) 0.8 % against 1.6.)
    const uint32_t in_range = (x.E & 255u) < 127u ? 0xffffffffu : 0u;
#pragma unroll
    for (int q = 0; q < 2; ++q) x.m[q] &= __vcmpne4(x.v[q], 0u) | in_range;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float2* th = reinterpret_cast<float2*>(&x.th[q]);
        const float2* gp = reinterpret_cast<const float2*>(&x.g[q]);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            float mo[2], vo[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t cm = byte_at_16(x.m[q] & 0x7f7f7f7fu, 2 * p + i), cv = byte_at_16(x.v[q], 2 * p + i);
                const uint32_t sign = __byte_perm(x.m[q], 0, 0x0444 + ((2 * p + i) << 12)) & 0x80000000u;
                mo[i] = __uint_as_float((cm ? cm * 16u + bm : 0u) | sign);
                vo[i] = __uint_as_float(cv ? cv * 16u + bv : 0u);
            }
            // products and sums rounded one by one: the same bits wherever this is computed
            const float2 g = mul_rn(make_float2(h.gscale, h.gscale), gp[p]);
            const float2 m = add_rn(mul_rn(make_float2(h.b1, h.b1), make_float2(mo[0], mo[1])), mul_rn(make_float2(h.one_b1, h.one_b1), g));
            const float2 v = add_rn(mul_rn(make_float2(h.b2, h.b2), make_float2(vo[0], vo[1])), mul_rn(mul_rn(make_float2(h.one_b2, h.one_b2), g), g));
            // theta -= lr (c1 m / (sqrt(c2 v) + eps) + wd theta), root and reciprocal to about an ulp of the step
            const float2 u = __fmul2_rn(m, make_float2(h.lr_c1, h.lr_c1));
            th[p].x = fmaf(-h.lr_wd, th[p].x, th[p].x) - u.x * rcp_approx(fmaf(sqrt_approx(v.x), h.sqrt_c2, h.eps));
            th[p].y = fmaf(-h.lr_wd, th[p].y, th[p].y) - u.y * rcp_approx(fmaf(sqrt_approx(v.y), h.sqrt_c2, h.eps));
            const int k = 4 * q + 2 * p;
            mb[k] = __float_as_uint(m.x);
            mb[k + 1] = __float_as_uint(m.y);
            vb[k] = __float_as_uint(v.x) & 0x7fffffffu;
            vb[k + 1] = __float_as_uint(v.y) & 0x7fffffffu;
            top_m = max(top_m, max(mb[k] & 0x7fffffffu, mb[k + 1] & 0x7fffffffu));
            top_v = max(top_v, max(vb[k], vb[k + 1]));
        }
        const int e = 128 * q + 4 * lane;
        if (e < left) {
            if (vec) {
                __stcs(reinterpret_cast<float4*>(theta + e), x.th[q]);
            } else {
                theta[e] = x.th[q].x; theta[e + 1] = x.th[q].y; theta[e + 2] = x.th[q].z; theta[e + 3] = x.th[q].w;
            }
        }
    }
    top_m = __reduce_max_sync(0xffffffffu, top_m);
    top_v = __reduce_max_sync(0xffffffffu, top_v);
    if (max(top_m, top_v) > OC_LARGEST) {
        top_m = top_v = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t a = magnitude(mb[k] & 0x7fffffffu);
            mb[k] = a | (__uint_as_float(mb[k]) < 0.f ? 0x80000000u : 0u);
            vb[k] = magnitude(vb[k]);
            top_m = max(top_m, a);
            top_v = max(top_v, vb[k]);
        }
        top_m = __reduce_max_sync(0xffffffffu, top_m);
        top_v = __reduce_max_sync(0xffffffffu, top_v);
    }
    const uint32_t Em = block_exponent(top_m), Ev = block_exponent(top_v);
    const uint32_t nm = code_base(Em, OC_M_ORDERS) << 20, nv = code_base(Ev, OC_V_ORDERS) << 20;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        int32_t cm[4], cv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = 4 * q + i;
            // mix32's last step leaves the high half as it is and adds it to the low half
            const uint32_t r = mix32_open(rnd + 4 * lane + (uint32_t)(128 * q + i)), high = r >> 16;
            cm[i] = code_of(mb[k] & 0x7fffffffu, (r ^ high) & 0xffffu, nm);
            cv[i] = max(code_of(vb[k], high, nv), (int32_t)min(vb[k], 1u));       // a positive v keeps the smallest code
        }
        // (a sign without a magnitude, of a -0 or a moment that was cut off, is a zero too)
        reinterpret_cast<uint32_t*>(blk)[32 * q + lane] = bytes(cm[0], cm[1], cm[2], cm[3]) | signs(mb[4 * q], mb[4 * q + 1], mb[4 * q + 2], mb[4 * q + 3]);
        reinterpret_cast<uint32_t*>(blk + 256)[32 * q + lane] = bytes(cv[0], cv[1], cv[2], cv[3]);
    }
    if (lane == 0) *reinterpret_cast<uint16_t*>(blk + 512) = (uint16_t)(Em | (Ev << 8));
}

// Rows of A per CTA: whole state blocks, at least 64 rows (128-byte runs of the pool's At rows) and `unit` elements.
__host__ __device__ __forceinline__ int rows_per_cta(int r, int unit) {
    int g = r, b = OC_BLOCK;        // 256 / gcd(256, r) rows are whole blocks
    while (b) {
        const int c = g % b;
        g = b;
        b = c;
    }
    const int step = OC_BLOCK / g, want = max(64, (unit + r - 1) / r);
    return (want + step - 1) / step * step;
}
__host__ __device__ __forceinline__ int tile_pitch(int r) { return r | 1; }     // odd: column reads spread over the banks

__device__ __forceinline__ int64_t state_bytes(int64_t n) { return (n + OC_BLOCK - 1) / OC_BLOCK * OC_STATE_BYTES; }

// One CTA per unit: a run of B, stored as the pool stores it, or a tile of rows of A, which goes through shared memory so
// that both the reads of A [K][r] and the writes of the pool's At rows [r][K] are contiguous.
template <int N>
__global__ void __launch_bounds__(OC_THREADS, 3) k_adamw_compact(const __grid_constant__ CompactArgs<N> a) {
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
    if (is_b) {
        int p = 0;
        int64_t soff = 0;
        for (; p < a.P - 1; ++p) {
            const int64_t n = (int64_t)r * (a.part_begin[p + 1] - a.part_begin[p]);
            const int units = (int)((n + a.unit - 1) / a.unit);
            if (u < units) break;
            u -= units;
            soff += state_bytes(n);
        }
        const int64_t c0 = a.part_begin[p], Np = a.part_begin[p + 1] - c0, n = (int64_t)r * Np;
        const uint32_t key = t.key[2 * p + 1];
        const float* grad = t.dB + (int64_t)r * c0;
        float* theta = t.B + (int64_t)r * c0;
        uint8_t* state = t.sB + soff;
        bf16* bs = a.Bs + (size_t)t.slot * a.RP * a.ldB + c0;
        const int64_t u0 = (int64_t)u * a.unit;
        const int count = (int)min((int64_t)a.unit, n - u0);
        grad += u0;
        theta += u0;
        state += u0 / OC_BLOCK * OC_STATE_BYTES;
        // the unit begins in row j0 at column i0.  Rows longer than a unit: at most one ends in it; else e / Np is the high
        // word of e over_n, both below 2^16
        const int64_t j0 = u0 / Np;
        const uint32_t i0 = (uint32_t)(u0 - j0 * Np), width = (uint32_t)Np;
        const bool wide = Np >= a.unit;
        const uint32_t over_n = wide ? 0u : 0xffffffffu / width + 1u;
        bs += j0 * a.ldB;
        // the next block's loads are under way while this one's step is computed
        constexpr int STEP = OC_THREADS / 32 * OC_BLOCK;
        CompactLane next;
        auto load = [&](int b) { compact_load(next, grad + b, theta + b, state + b / OC_BLOCK * OC_STATE_BYTES, count - b, vec, lane); };
        if (warp * OC_BLOCK < count) load(warp * OC_BLOCK);
        for (int b = warp * OC_BLOCK; b < count; b += STEP) {
            CompactLane x = next;
            uint8_t* blk = state + b / OC_BLOCK * OC_STATE_BYTES;
            if (b + STEP < count) load(b + STEP);
            compact_step(x, a.h, theta + b, blk, count - b, vec, (uint32_t)u0 + (uint32_t)b + key, lane);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int e = b + 128 * q + 4 * lane;
                if (e >= count) continue;
                const uint32_t c = i0 + (uint32_t)e, dj = wide ? (uint32_t)(c >= width) : __umulhi(c, over_n);   // four elements of one row
                __nv_bfloat162 y = __floats2bfloat162_rn(x.th[q].x, x.th[q].y), z = __floats2bfloat162_rn(x.th[q].z, x.th[q].w);
                *reinterpret_cast<uint2*>(bs + (int64_t)dj * a.ldB + (c - dj * width)) =
                    make_uint2(*reinterpret_cast<uint32_t*>(&y), *reinterpret_cast<uint32_t*>(&z));
            }
        }
        return;
    }
    const int R = rows_per_cta(r, a.unit), pitch = tile_pitch(r);
    const int per_part = (int)((a.K + R - 1) / R);
    const int p = u / per_part;
    const int64_t k0 = (int64_t)(u - p * per_part) * R, n = a.K * r, poff = (int64_t)p * n;
    const int rows = (int)min((int64_t)R, a.K - k0), elems = rows * r;
    const uint32_t key = t.key[2 * p], over_r = r > 1 ? 0xffffffffu / (uint32_t)r + 1u : 0u;      // e / r = high word of e over_r (e < 2^16)
    const float* grad = t.dA + poff + k0 * r;
    float* theta = t.A + poff + k0 * r;
    uint8_t* state = t.sA + p * state_bytes(n) + k0 * r / OC_BLOCK * OC_STATE_BYTES;
    constexpr int STEP = OC_THREADS / 32 * OC_BLOCK;
    CompactLane next;
    auto load = [&](int b) { compact_load(next, grad + b, theta + b, state + b / OC_BLOCK * OC_STATE_BYTES, elems - b, vec, lane); };
    if (warp * OC_BLOCK < elems) load(warp * OC_BLOCK);
    for (int b = warp * OC_BLOCK; b < elems; b += STEP) {
        CompactLane x = next;
        uint8_t* blk = state + b / OC_BLOCK * OC_STATE_BYTES;
        if (b + STEP < elems) load(b + STEP);
        compact_step(x, a.h, theta + b, blk, elems - b, vec, (uint32_t)(k0 * r) + (uint32_t)b + key, lane);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = b + 128 * q + 4 * lane;
            if (e >= elems) continue;
            int kk = r > 1 ? (int)__umulhi((uint32_t)e, over_r) : e, j = e - kk * r;
            bf16* to = tile + kk * pitch + j;
            if ((r & 3) == 0) {         // four elements of one row
                to[0] = __float2bfloat16_rn(x.th[q].x);
                to[1] = __float2bfloat16_rn(x.th[q].y);
                to[2] = __float2bfloat16_rn(x.th[q].z);
                to[3] = __float2bfloat16_rn(x.th[q].w);
            } else {
                const float th[4] = {x.th[q].x, x.th[q].y, x.th[q].z, x.th[q].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *to++ = __float2bfloat16_rn(th[i]);
                    if (++j == r) {
                        j = 0;
                        to += pitch - r;
                    }
                }
            }
        }
    }
    __syncthreads();
    // A thread takes 8 rows of a column; neighbours take neighbouring columns (conflict-free reads of the tile), so that a
    // warp's 16-byte writes go to as many rows of At and the lines fill up in L2.  K and R are multiples of 8.
    bf16* at = a.At + ((size_t)p * a.cap + t.slot) * a.RP * (size_t)a.K + k0;
    const int work = rows / 8 * r;
    for (int x = tid; x < work; x += OC_THREADS) {
        const int g = r > 1 ? (int)__umulhi((uint32_t)x, over_r) : x, j = x - g * r;
        const bf16* from = tile + 8 * g * pitch + j;
        uint4 o;
        uint32_t* w = &o.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 y;
            y.x = from[2 * i * pitch];
            y.y = from[(2 * i + 1) * pitch];
            w[i] = *reinterpret_cast<uint32_t*>(&y);
        }
        *reinterpret_cast<uint4*>(at + (size_t)j * a.K + 8 * g) = o;
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
        const uint32_t bm = code_base(E & 255u, OC_M_ORDERS) << 20, bv = code_base(E >> 8, OC_V_ORDERS) << 20;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t mc = reinterpret_cast<const uint32_t*>(blk)[32 * q + lane];
            const uint32_t vc = reinterpret_cast<const uint32_t*>(blk + 256)[32 * q + lane];
            float fm[4], fv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = byte_of(mc, i);
                fm[i] = __uint_as_float(__float_as_uint(code_value(c & 127u, bm)) | ((c & 128u) << 24));
                fv[i] = code_value(byte_of(vc, i), bv);
            }
            const int64_t e = b * OC_BLOCK + 128 * q + 4 * lane;
            if (m) *reinterpret_cast<float4*>(m + e) = make_float4(fm[0], fm[1], fm[2], fm[3]);
            if (v) *reinterpret_cast<float4*>(v + e) = make_float4(fv[0], fv[1], fv[2], fv[3]);
        }
    }
}

template <int N>
static marlaas_status_t launch_compact(const marlaas_pool* pool, const CompactTenant* t, int n, const marlaas_adamw_t& hp, cudaStream_t st) {
    CompactArgs<N> a;
    a.n = n; a.P = pool->P; a.RP = pool->RP; a.cap = pool->cap; a.K = pool->K; a.ldB = pool->ldB;
    for (int p = 0; p <= MARLAAS_MAX_PARTS; ++p) a.part_begin[p] = pool->part_begin[p];
    const double c1 = 1.0 / (1.0 - std::pow((double)hp.beta1, (double)hp.step)), c2 = 1.0 / (1.0 - std::pow((double)hp.beta2, (double)hp.step));
    a.h.b1 = hp.beta1; a.h.b2 = hp.beta2; a.h.one_b1 = 1.f - hp.beta1; a.h.one_b2 = 1.f - hp.beta2; a.h.gscale = hp.grad_scale;
    a.h.sqrt_c2 = (float)std::sqrt(c2); a.h.eps = hp.eps; a.h.lr_c1 = (float)(hp.lr * c1); a.h.lr_wd = hp.lr * hp.weight_decay;
    // Longer units spread a CTA's set-up over more elements and overlap more loads with steps, shorter ones spread a small update
    // over more SMs.  32 tenants of ranks 8 to 64, 32 and 16, us with short / long units: 0.5 M elements 6.3-8.3 / 10.1-10.3,
    // 1 M 10.4-11.4 / 10.4-12.4, 2 M 14.5-14.9 / 13.1-16.5, 3 M 18.6-19.0 / 16.5-17.4, 5 M 26.8 / 24.6-24.9, 10 M 47-48 / 39-40,
    // 25 M 107-113 / 84-85.  The change is at two long units per SM, 2.4 M elements.
    int64_t elems = 0;
    for (int i = 0; i < n; ++i) elems += t[i].rank * (pool->P * pool->K + pool->N);
    a.unit = elems >= (int64_t)pool->sm_count * 2 * OC_UNIT * OC_LONG ? OC_UNIT * OC_LONG : OC_UNIT;
    a.At = pool->d_At; a.Bs = pool->d_Bs;
    int64_t ctas = 0;
    size_t smem = 0;
    for (int i = 0; i < n; ++i) {
        const int r = t[i].rank, R = rows_per_cta(r, a.unit);
        a.t[i] = t[i];
        a.first[2 * i] = (int32_t)ctas;
        ctas += (int64_t)pool->P * cdiv(pool->K, R);
        a.first[2 * i + 1] = (int32_t)ctas;
        for (int p = 0; p < pool->P; ++p) ctas += cdiv((int64_t)r * (pool->part_begin[p + 1] - pool->part_begin[p]), (int64_t)a.unit);
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
        t[i] = CompactTenant{dA[i], dB[i], A[i], B[i], (uint8_t*)state_A[i], (uint8_t*)state_B[i], slot,
                             (uint16_t)pool->slots[slot].rank, (uint16_t)((low & 15) == 0), {}};
        for (uint32_t k = 0; k < 2u * pool->P; ++k) t[i].key[k] = stream_key(seed, (uint64_t)hp->step, tenant_ids[i], k);
    }
    MARLAAS_CUDA_TRY(cudaSetDevice(pool->device));
    for (int i0 = 0; i0 < n; i0 += OC_MAX_TENANTS) {
        const int m = std::min(OC_MAX_TENANTS, n - i0);
        marlaas_status_t rc = m <= 8    ? launch_compact<8>(pool, t.data() + i0, m, *hp, (cudaStream_t)cuda_stream)
                              : m <= 48 ? launch_compact<48>(pool, t.data() + i0, m, *hp, (cudaStream_t)cuda_stream)
                                        : launch_compact<OC_MAX_TENANTS>(pool, t.data() + i0, m, *hp, (cudaStream_t)cuda_stream);
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
