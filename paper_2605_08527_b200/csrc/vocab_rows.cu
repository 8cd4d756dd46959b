// Rows of logits: log-probability of the target, entropy, the clipped policy loss's terms and the gradient by the logits
// (Algorithm 1: "PolicyUpdate"; Experimental setup: GRPO).  With z the row, k = inv_temperature:
//     m = max z    s = sum exp((z - m) k)    logp = (z_a - m) k - log s    H = log s - sum p (z - m) k
//     dz_j = g ( p_j (c_H (log p_j + H) - c) + [j = a] c ),   g = grad_scale w k,   c = d(pg + kl_coef kl) / d logp
#include <math_constants.h>

#include "sm100_ptx.cuh"

namespace marlaas {

constexpr int VR_THREADS = 512;
constexpr float VR_LOG2E = 1.4426950408889634f, VR_LN2 = 0.6931471805599453f;

// max that keeps a NaN (fmaxf drops it): a bad logit has to show in the row's outputs
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The reference point of a running maximum: 0 while there is no finite logit, so that -inf - m stays -inf.
__device__ __forceinline__ float ref_of(float m) { return m == -CUDART_INF_F ? 0.f : m; }
// (z - m) k in units of log 2, not below -200: 2^-200 is 0 in fp32, and a product with it stays 0 where (z - m) k itself is
// -inf.  The difference comes first: z k alone may leave fp32's range where a mask is the type's lowest value.
__device__ __forceinline__ float exponent(float z, float m, float k2) { return max_nan((z - m) * k2, -200.f); }

struct RowStats {       // running statistics of a part of a row, relative to its own maximum
    float m, s, u;      // u = sum 2^t t, t = exponent of each element
};
__device__ __forceinline__ RowStats merge(RowStats a, RowStats b, float k2) {
    RowStats r;
    r.m = max_nan(a.m, b.m);
    const float mr = ref_of(r.m);
    const float da = exponent(a.m, mr, k2), db = exponent(b.m, mr, k2);
    const float fa = ex2(da), fb = ex2(db);
    r.s = fa * a.s + fb * b.s;
    r.u = fa * (a.u + a.s * da) + fb * (b.u + b.s * db);
    return r;
}

template <bool F32>
struct Vec;
template <>
struct Vec<false> {     // 8 bf16 in 16 bytes
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(uint4 q, float (&f)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        uint4 q;
        uint32_t* w = &q.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
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
    static __device__ __forceinline__ void unpack(uint4 q, float (&f)[4]) {
        f[0] = __uint_as_float(q.x); f[1] = __uint_as_float(q.y); f[2] = __uint_as_float(q.z); f[3] = __uint_as_float(q.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float load(const void* p, int64_t i) { return ((const float*)p)[i]; }
    static __device__ __forceinline__ void store(void* p, int64_t i, float v) { ((float*)p)[i] = v; }
};

// What a row's gradient needs: dz_j = 2^(t_j - log2 s) (alpha t_j + beta), and + gamma at the target.
struct RowGrad {
    float alpha, beta, gamma;
};

// The token's loss terms from its log-probability and entropy; the coefficients of its gradient.
__device__ __forceinline__ RowGrad token_terms(const VocabRows& a, int64_t i, float logp, float H, float log2s, PolicyTerms* out) {
    const float w = a.weight[i], A = a.adv[i];
    const float ratio = expf(logp - a.old_logp[i]);
    // 0 A is 0 whatever the ratio
    const float plain = A == 0.f ? 0.f : ratio * A;
    const float clipped = A == 0.f ? 0.f : fminf(fmaxf(ratio, 1.f - a.clip_low), 1.f + a.clip_high) * A;
    const bool is_clipped = plain > clipped;      // (a NaN counts as not clipped and shows in the loss)
    const float pg = -(is_clipped ? clipped : plain);
    float c = is_clipped ? 0.f : -plain, kl = 0.f;
    if (a.kl_coef != 0.f) {
        const float d = a.ref_logp[i] - logp, e1 = expm1f(d);     // exp(d) - d - 1 without its cancellation for small d
        kl = e1 - d;
        c -= a.kl_coef * e1;
    }
    PolicyTerms t;
    t.loss = w * (pg + a.kl_coef * kl - a.entropy_coef * H);
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

// One CTA per row, which is read twice: statistics, then the gradient.
template <bool F32>
__global__ void __launch_bounds__(VR_THREADS) k_vocab_rows(const VocabRows a) {
    using X = Vec<F32>;
    constexpr int E = F32 ? 4 : 2;
    __shared__ RowStats s_part[VR_THREADS / 32];
    __shared__ RowGrad s_grad;
    __shared__ float s_log2s, s_m;
    __shared__ int s_live;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float k2 = a.inv_temperature * VR_LOG2E;
    const int64_t V = a.V, nv = V / X::N;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        const char* z = (const char*)a.logits + (size_t)row * a.ld * E;
        char* dz = a.dlogits ? (char*)a.dlogits + (size_t)row * a.lddl * E : nullptr;
        const int32_t target = a.targets[row];
        bool live = target >= 0 && target < V;
        if (target >= V && tid == 0) {
            if (atomicCAS(a.status, 0, DEV_BAD_INDEX) == 0) a.status[1] = (int)row;
        }
        const bool wanted = !a.terms || a.weight[row] != 0.f;      // else only logp / entropy
        if (live && (wanted || a.logp || a.entropy)) {
            RowStats st = {-CUDART_INF_F, 0.f, 0.f};
            for (int64_t v = tid; v < nv; v += VR_THREADS) {
                float f[X::N];
                X::unpack(reinterpret_cast<const uint4*>(z)[v], f);
                RowStats b = {f[0], 0.f, 0.f};
#pragma unroll
                for (int i = 1; i < X::N; ++i) b.m = max_nan(b.m, f[i]);
                const float mr = ref_of(b.m);
#pragma unroll
                for (int i = 0; i < X::N; ++i) {
                    const float t = exponent(f[i], mr, k2), e = ex2(t);
                    b.s += e;
                    b.u += e * t;
                }
                st = merge(st, b, k2);
            }
            for (int64_t i = nv * X::N + tid; i < V; i += VR_THREADS) {
                const float f = X::load(z, i);
                const float t = exponent(f, ref_of(f), k2), e = ex2(t);
                st = merge(st, RowStats{f, e, e * t}, k2);
            }
            for (int o = 16; o > 0; o >>= 1) {
                RowStats b;
                b.m = __shfl_xor_sync(0xffffffffu, st.m, o);
                b.s = __shfl_xor_sync(0xffffffffu, st.s, o);
                b.u = __shfl_xor_sync(0xffffffffu, st.u, o);
                st = merge(st, b, k2);
            }
            if (lane == 0) s_part[warp] = st;
            __syncthreads();
            if (tid == 0) {
                for (int w = 1; w < VR_THREADS / 32; ++w) st = merge(st, s_part[w], k2);
                const bool dist = !(st.s == 0.f);
                const float log2s = dist ? log2f(st.s) : 0.f, mr = ref_of(st.m);
                const float logp = dist ? ((X::load(z, target) - mr) * k2 - log2s) * VR_LN2 : 0.f;
                const float H = dist ? (log2s - st.u / st.s) * VR_LN2 : 0.f;
                if (a.logp) a.logp[row] = logp;
                if (a.entropy) a.entropy[row] = H;
                s_live = dist && wanted;
                s_m = mr;
                s_log2s = log2s;
                if (a.terms && s_live) s_grad = token_terms(a, row, logp, H, log2s, a.terms + row);
            }
            __syncthreads();
            live = s_live;
        } else {
            if (tid == 0) {
                if (a.logp) a.logp[row] = 0.f;
                if (a.entropy) a.entropy[row] = 0.f;
            }
            live = false;
        }
        if (a.terms && !live && tid == 0) a.terms[row] = PolicyTerms{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (dz) {
            if (!live) {
                for (int64_t v = tid; v < nv; v += VR_THREADS) reinterpret_cast<uint4*>(dz)[v] = make_uint4(0, 0, 0, 0);
                for (int64_t i = nv * X::N + tid; i < V; i += VR_THREADS) X::store(dz, i, 0.f);
            } else {
                const RowGrad g = s_grad;
                const float m = s_m, log2s = s_log2s;
                for (int64_t v = tid; v < nv; v += VR_THREADS) {
                    float f[X::N];
                    X::unpack(reinterpret_cast<const uint4*>(z)[v], f);
#pragma unroll
                    for (int i = 0; i < X::N; ++i) {
                        const float t = exponent(f[i], m, k2);
                        f[i] = ex2(t - log2s) * (g.alpha * t + g.beta);
                        if (v * X::N + i == target) f[i] += g.gamma;
                    }
                    reinterpret_cast<uint4*>(dz)[v] = X::pack(f);
                }
                for (int64_t i = nv * X::N + tid; i < V; i += VR_THREADS) {
                    const float t = exponent(X::load(z, i), m, k2);
                    X::store(dz, i, ex2(t - log2s) * (g.alpha * t + g.beta) + (i == target ? g.gamma : 0.f));
                }
            }
        }
        __syncthreads();
    }
}

marlaas_status_t launch_vocab_rows(const marlaas_pool* pool, const VocabRows& r, cudaStream_t st) {
    const int grid = (int)std::min<int64_t>(r.T, (int64_t)pool->sm_count * 4);
    if (r.f32) k_vocab_rows<true><<<grid, VR_THREADS, 0, st>>>(r);
    else k_vocab_rows<false><<<grid, VR_THREADS, 0, st>>>(r);
    MARLAAS_LAUNCH_CHECK("k_vocab_rows");
    return MARLAAS_OK;
}

}  // namespace marlaas
