// Losses on logits with their gradients: distillation from a teacher's top logits, the clipped policy
// loss, and the log-probabilities, pairs and gradient of the preference loss.
//
// A row's statistics are the running maximum m and sums s = sum exp((z - m) / tau) of a softmax;
// log p_v = (z_v - m) / tau - log s and p_v = exp((z_v - m) / tau) / s.  Everything is formed from
// z - m, so logits of the type's lowest value and of -infinity need no special case: m is taken as 0
// where every logit is -infinity (then s = 0: the row leaves no distribution), and a NaN reaches s.
#include <math_constants.h>

#include "glr_loss.cuh"

namespace glr {
namespace loss {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float load(const float* p) { return *p; }
__device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Maximum, and sums of exp at two temperatures (s1: temperature 1, for a hard term beside tau != 1).
struct Stat { float m, s, s1; };
// Teacher: maximum, sum of e = exp((a - m) / tau), sums of e a and e (z_id - the row's maximum).
struct Top { float m, s, a, z; };

// exp2((a - m) c) for a <= m, with exp of -infinity against -infinity counted as 1 (its sum is 0)
__device__ __forceinline__ float shrink(float a, float m, float c) {
    return a == -CUDART_INF_F ? 1.f : exp2_fast((a - m) * c);
}
__device__ __forceinline__ Stat merge(const Stat& x, const Stat& y, float c) {
    Stat r;
    r.m = fmaxf(x.m, y.m);
    r.s = x.s * shrink(x.m, r.m, c) + y.s * shrink(y.m, r.m, c);
    r.s1 = x.s1 * shrink(x.m, r.m, kLog2e) + y.s1 * shrink(y.m, r.m, kLog2e);
    return r;
}
__device__ __forceinline__ Top merge(const Top& x, const Top& y, float c) {
    Top r;
    r.m = fmaxf(x.m, y.m);
    const float fx = shrink(x.m, r.m, c), fy = shrink(y.m, r.m, c);
    r.s = x.s * fx + y.s * fy;
    r.a = x.a * fx + y.a * fy;
    r.z = x.z * fx + y.z * fy;
    return r;
}
__device__ __forceinline__ Stat shuffle(const Stat& x, int d) {
    return {__shfl_xor_sync(~0u, x.m, d), __shfl_xor_sync(~0u, x.s, d), __shfl_xor_sync(~0u, x.s1, d)};
}
__device__ __forceinline__ Top shuffle(const Top& x, int d) {
    return {__shfl_xor_sync(~0u, x.m, d), __shfl_xor_sync(~0u, x.s, d), __shfl_xor_sync(~0u, x.a, d),
            __shfl_xor_sync(~0u, x.z, d)};
}
// The block's merge, in a fixed order, to every thread.
template <class S>
__device__ S block_merge(S x, float c, S* scratch) {
    for (int d = 16; d; d >>= 1) x = merge(x, shuffle(x, d), c);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    S r = scratch[0];
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) r = merge(r, scratch[w], c);
    return r;
}

constexpr int kThreads = 512;

// One CTA a row, the row read twice (statistics, gradient).
template <int K, class T>
__global__ void __launch_bounds__(kThreads) rows_kernel(const RowArgs a) {
    chain_begin();
    __shared__ Stat stat_s[kThreads / 32];
    __shared__ Top top_s[kThreads / 32];
    __shared__ int32_t id_s[GLR_MAX_TOPK + 1];
    __shared__ float q_s[GLR_MAX_TOPK + 1];
    const float c = a.inv_tau * kLog2e;
    const int tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + row * a.ldz;
        T* dz = a.dz ? static_cast<T*>(a.dz) + row * a.lddz : nullptr;
        const float w = a.weight ? a.weight[row] : a.share;
        int64_t tok = -1;
        if (K != kDistill) tok = a.tokens.at(row);
        else if (a.labels.p) tok = a.labels.at(row);
        const bool has_tok = tok >= 0 && tok < a.vocab;
        bool counts = K == kDistill ? w != 0.f : K == kPolicy ? has_tok && w != 0.f : has_tok;
        Stat st{-CUDART_INF_F, 0.f, 0.f};
        if (counts) {
            for (int64_t v = tid; v < a.vocab; v += kThreads) {
                const float x = load(z + v);
                const float m = fmaxf(st.m, x), r = m == -CUDART_INF_F ? 0.f : m;
                st.s = st.s * shrink(st.m, m, c) + exp2_fast((x - r) * c);
                if (K == kDistill) st.s1 = st.s1 * shrink(st.m, m, kLog2e) + exp2_fast((x - r) * kLog2e);
                st.m = m;
            }
        }
        st = block_merge(st, c, stat_s);
        if (st.s == 0.f) counts = false;
        const float ln_s = logf(st.s);
        float dense = 0.f, dense1 = 0.f;     // factors of exp2((z - m) c) and exp2((z - m) log2 e)
        int n = 0;                            // entries subtracted at their ids
        if (K == kDistill) {
            Top tp{-CUDART_INF_F, 0.f, 0.f, 0.f};
            float aval[GLR_MAX_TOPK / kThreads];
#pragma unroll
            for (int u = 0; u < GLR_MAX_TOPK / kThreads; ++u) {
                const int k = tid + u * kThreads;
                int64_t id = -1;
                aval[u] = -CUDART_INF_F;
                if (k < a.topk) {
                    id = a.ids.at(row * a.ldi + k);
                    if (id >= a.vocab) id = -1;
                    if (id >= 0 && counts) {
                        const int64_t at = row * a.ldt + k;
                        aval[u] = a.teacher_bf16 ? load(static_cast<const __nv_bfloat16*>(a.teacher) + at)
                                                 : static_cast<const float*>(a.teacher)[at];
                        // an entry ruled out by the teacher leaves the sums as they are
                        if (aval[u] != -CUDART_INF_F) tp = merge(tp, Top{aval[u], 1.f, aval[u], load(z + id) - st.m}, c);
                    }
                    id_s[k] = static_cast<int32_t>(id);
                }
            }
            tp = block_merge(tp, c, top_s);
            const bool soft = counts && tp.s != 0.f, hard = counts && has_tok && a.labels.p;
            float loss = 0.f;
            if (soft) {
                const float ln_st = logf(tp.s), inv = 1.f / tp.s;
                loss = a.soft * (((tp.a * inv - tp.m) * a.inv_tau - ln_st) - (tp.z * inv * a.inv_tau - ln_s));
                dense = w * a.soft * a.inv_tau / st.s;
            }
#pragma unroll
            for (int u = 0; u < GLR_MAX_TOPK / kThreads; ++u) {
                const int k = tid + u * kThreads;
                if (k < a.topk) q_s[k] = soft ? w * a.soft * a.inv_tau * shrink(aval[u], tp.m, c) / tp.s : 0.f;
                if (k < a.topk && aval[u] == -CUDART_INF_F) q_s[k] = 0.f;
            }
            n = soft ? a.topk : 0;
            if (hard) {
                loss += a.hard * -((load(z + tok) - st.m) - logf(st.s1));
                dense1 = w * a.hard / st.s1;
                if (tid == 0) { id_s[n] = static_cast<int32_t>(tok); q_s[n] = w * a.hard; }
                ++n;
            }
            if (tid == 0) a.row_loss[row] = loss;
        } else {
            const float lp = counts ? (load(z + tok) - st.m) * a.inv_tau - ln_s : 0.f;
            if (K == kPolicy) {
                float loss = 0.f, slope = 0.f;
                if (counts) {
                    const float A = a.advantage[row], ratio = expf(lp - a.old_logp[row]);
                    loss = -fminf(ratio * A, fminf(fmaxf(ratio, a.clip_lo), a.clip_hi) * A);
                    if (isnan(ratio * A)) loss = ratio * A;
                    slope = (A > 0.f ? ratio > a.clip_hi : ratio < a.clip_lo) ? 0.f : -A * ratio;
                    if (a.ref_logp) {
                        const float e = expm1f(a.ref_logp[row] - lp);
                        loss += a.kl * (e - (a.ref_logp[row] - lp));
                        slope -= a.kl * e;
                    }
                }
                const float coef = slope * w * a.inv_tau;
                dense = counts ? -coef / st.s : 0.f;
                if (counts) { n = 1; if (tid == 0) { id_s[0] = static_cast<int32_t>(tok); q_s[0] = -coef; } }
                if (tid == 0) { a.row_loss[row] = loss; a.logp[row] = lp; }
            } else if (tid == 0) {
                a.logp[row] = lp;
                a.lse[row] = counts ? st.m + ln_s : CUDART_INF_F;
                a.coef[row] = 0.f;
            }
        }
        if (K != kLogProb && dz) {
            __syncthreads();
            // the gradients at the listed ids are formed before the row is overwritten (dz may be z)
            float mine[GLR_MAX_TOPK / kThreads + 1];
#pragma unroll
            for (int u = 0; u <= GLR_MAX_TOPK / kThreads; ++u) {
                const int k = tid + u * kThreads;
                mine[u] = 0.f;
                if (k < n && id_s[k] >= 0) {
                    const float x = load(z + id_s[k]);
                    float g = 0.f;
                    for (int j = 0; j < n; ++j) g += id_s[j] == id_s[k] ? q_s[j] : 0.f;
                    mine[u] = dense * exp2_fast((x - st.m) * c) + dense1 * exp2_fast((x - st.m) * kLog2e) - g;
                }
            }
            __syncthreads();
            for (int64_t v = tid; v < a.vocab; v += kThreads) {
                float g = 0.f;
                if (counts) {
                    const float x = load(z + v) - st.m;
                    g = dense * exp2_fast(x * c);
                    if (K == kDistill && dense1 != 0.f) g += dense1 * exp2_fast(x * kLog2e);
                }
                store(dz + v, g);
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u <= GLR_MAX_TOPK / kThreads; ++u) {
                const int k = tid + u * kThreads;
                if (k < n && id_s[k] >= 0) store(dz + id_s[k], mine[u]);
            }
            __syncthreads();
        }
    }
}

// Sums of a sequence's log-probabilities in 64 bits, thread by thread and then up the same tree.
__device__ double block_sum(double x, double* scratch) {
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    double r = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) r += scratch[w];
    return r;
}

constexpr int kPairThreads = 256;
// One CTA a pair.
__global__ void __launch_bounds__(kPairThreads) pairs_kernel(const PairArgs a) {
    chain_begin();
    __shared__ double scratch[kPairThreads / 32];
    const int64_t p = blockIdx.x;
    int64_t at[2][2];
    float seq[2], share[2];
    for (int h = 0; h < 2; ++h) {
        int64_t b = a.offsets.at(2 * p + h), e = a.offsets.at(2 * p + h + 1);
        b = b < 0 ? 0 : b > a.rows ? a.rows : b;
        e = e < b ? b : e > a.rows ? a.rows : e;
        at[h][0] = b; at[h][1] = e;
        double sum = 0, cnt = 0;
        for (int64_t t = b + threadIdx.x; t < e; t += kPairThreads) {
            sum += a.row_logp[t];
            cnt += a.lse[t] != CUDART_INF_F;
        }
        sum = block_sum(sum, scratch);
        share[h] = 1.f;
        if (a.average) {
            cnt = block_sum(cnt, scratch);
            share[h] = static_cast<float>(1.0 / (cnt < 1 ? 1 : cnt));
            sum /= cnt < 1 ? 1 : cnt;
        }
        seq[h] = static_cast<float>(sum);
    }
    const float w = a.weight ? a.weight[p] : a.share;
    const float h = (seq[0] - (a.ref_logp ? a.ref_logp[2 * p] : 0.f)) - (seq[1] - (a.ref_logp ? a.ref_logp[2 * p + 1] : 0.f));
    float loss, slope;
    if (a.kind == GLR_PREF_IPO) {
        const float e = h - 0.5f / a.beta;
        loss = e * e;
        slope = 2.f * e;
    } else {
        // -log sigmoid(x) = max(-x, 0) + log1p(exp(-|x|))
        const float x = a.beta * h, t = log1pf(expf(-fabsf(x)));
        loss = (1.f - a.smoothing) * (fmaxf(-x, 0.f) + t) + a.smoothing * (fmaxf(x, 0.f) + t);
        if (isnan(x)) loss = x;
        slope = a.beta * (a.smoothing / (1.f + expf(-x)) - (1.f - a.smoothing) / (1.f + expf(x)));
    }
    if (threadIdx.x == 0) {
        a.seq_logp[2 * p] = seq[0];
        a.seq_logp[2 * p + 1] = seq[1];
        a.pair_loss[p] = loss;
    }
    for (int s = 0; s < 2; ++s) {
        const float coef = w == 0.f ? 0.f : (s ? -slope : slope) * w * share[s];
        for (int64_t t = at[s][0] + threadIdx.x; t < at[s][1]; t += kPairThreads)
            if (a.lse[t] != CUDART_INF_F) a.coef[t] = coef;
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) grad_kernel(const RowArgs a) {
    chain_begin();
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + row * a.ldz;
        T* dz = static_cast<T*>(a.dz) + row * a.lddz;
        const float coef = a.coef[row], lse = a.lse[row];
        const int64_t tok = coef == 0.f ? -1 : a.tokens.at(row);
        for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) {
            float g = 0.f;
            if (coef != 0.f) {
                const float p = exp2_fast((load(z + v) - lse) * kLog2e);
                g = v == tok ? coef - coef * p : -coef * p;
            }
            store(dz + v, g);
        }
    }
}

constexpr int kTotalThreads = 1024;
__global__ void __launch_bounds__(kTotalThreads) total_kernel(const float* x, const float* weight, float share, int64_t n,
                                                              float* out) {
    chain_begin();
    __shared__ double scratch[kTotalThreads / 32];
    double s = 0;
    for (int64_t i = threadIdx.x; i < n; i += kTotalThreads) {
        const float w = weight ? weight[i] : share;
        if (w != 0.f) s += static_cast<double>(w) * x[i];
    }
    s = block_sum(s, scratch);
    if (threadIdx.x == 0) *out = static_cast<float>(s);
}

template <int K>
cudaError_t rows_launch(const RowArgs& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const int grid = static_cast<int>(a.rows < 152 * 4 ? a.rows : 152 * 4);
    return dtype == GLR_BF16 ? launch_chain(rows_kernel<K, __nv_bfloat16>, grid, kThreads, 0, st, a)
                             : launch_chain(rows_kernel<K, float>, grid, kThreads, 0, st, a);
}

}  // namespace

cudaError_t distill(const RowArgs& a, int dtype, cudaStream_t st) { return rows_launch<kDistill>(a, dtype, st); }
cudaError_t policy(const RowArgs& a, int dtype, cudaStream_t st) { return rows_launch<kPolicy>(a, dtype, st); }
cudaError_t log_prob(const RowArgs& a, int dtype, cudaStream_t st) { return rows_launch<kLogProb>(a, dtype, st); }

cudaError_t pairs(const PairArgs& a, cudaStream_t st) {
    if (a.pairs == 0) return cudaSuccess;
    return launch_chain(pairs_kernel, static_cast<unsigned>(a.pairs), kPairThreads, 0, st, a);
}

cudaError_t log_prob_grad(const RowArgs& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const int grid = static_cast<int>(a.rows < 152 * 4 ? a.rows : 152 * 4);
    return dtype == GLR_BF16 ? launch_chain(grad_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a)
                             : launch_chain(grad_kernel<float>, grid, kThreads, 0, st, a);
}

cudaError_t total(const float* x, const float* weight, float share, int64_t n, float* out, cudaStream_t st) {
    return launch_chain(total_kernel, 1, kTotalThreads, 0, st, x, weight, share, n, out);
}

}  // namespace loss
}  // namespace glr
