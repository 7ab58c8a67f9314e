// Log-probabilities of given tokens with the entropy and the most probable alternatives, and their gradient.
//
// With x_v = (z_v - m) / tau, m the row's maximum, s = sum e^x and u = sum e^x x:
//   lse = m / tau + log s,  logp = x_token - log s,  entropy = log s - u / s  (both terms are of one sign)
// A thread keeps a running maximum and rescales its sums when it grows.  Entries of -infinity add nothing to either sum, and a
// NaN reaches s.
// The alternatives are ordered by a 64-bit key: the logit as an integer of the same order (-0 as 0, a NaN above all) over the
// complement of its index, so that no two are equal and equal logits go by their index.
#include <algorithm>

#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A row's statistics over a part of its entries: maximum of the finite ones (kLowest: none), sums relative to it, in powers of two.
struct Stat { float m, s, u; };
// ... of two parts.  c = log2(e) / tau.
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float c) {
    const float m = fmaxf(a.m, b.m);
    // (an infinity is its own maximum: inf - inf is the NaN that the sums are then)
    const float da = (a.m - m) * c, db = (b.m - m) * c, ea = exp2_fast(da), eb = exp2_fast(db);
    Stat r;
    r.m = m;
    r.s = a.s * ea + b.s * eb;
    r.u = (a.s != 0.f ? (a.u + a.s * fmaxf(da, -1e30f)) * ea : 0.f) + (b.s != 0.f ? (b.u + b.s * fmaxf(db, -1e30f)) * eb : 0.f);
    return r;
}

// The logit as an integer of the same order; 0 for an entry that is ruled out.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);     // -0 is 0
    if (z != z) return 0xffffffffu;
    if (b == 0xff800000u) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t order) {
    if (order == 0xffffffffu) return __uint_as_float(0x7fffffffu);
    return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ uint64_t key_of(float z, uint32_t index) { return static_cast<uint64_t>(order_of(z)) << 32 | ~index; }

// A row as vectors of eight that begin on 16 bytes, the first one at or before the row's first element: `skip` elements of
// it are not the row's.  (Where elements are not on their vectors' pitch, as in rows of fp32 off 32 bytes, eight of fp32
// begin on 16 bytes too.)
template <class T>
struct RowVectors {
    const T* base;
    int skip;
    int64_t vocab, count;
    __device__ RowVectors(const T* z, int64_t v) : vocab(v) {
        skip = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
        base = z - skip;
        count = (skip + v + 7) / 8;
    }
    __device__ __forceinline__ int64_t first(int64_t q) const { return q * 8 - skip; }     // index of vector q's first element
    // -infinity where there is no element
    __device__ __forceinline__ void load(int64_t q, float (&v)[8]) const {
        const int64_t i = first(q);
        if (i >= 0 && i + 8 <= vocab) {
            load8(base + q * 8, 8, true, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = i + e >= 0 && i + e < vocab ? to_f(base[q * 8 + e]) : -__int_as_float(0x7f800000);
        }
    }
};

// The CTA's keys in descending order; n <= size, a power of two; the places behind are filled with 0.
__device__ __forceinline__ void sort_keys(uint64_t* key, int n, int size) {
    for (int q = n + threadIdx.x; q < size; q += kThreads) key[q] = 0;
    __syncthreads();
    for (int len = 2; len <= size; len *= 2)
        for (int gap = len / 2; gap > 0; gap /= 2) {
            for (int q = threadIdx.x; q < size / 2; q += kThreads) {
                const int i = 2 * q - (q & (gap - 1)), j = i + gap;
                const uint64_t x = key[i], y = key[j];
                if ((x < y) == ((i & len) == 0)) { key[i] = y; key[j] = x; }
            }
            __syncthreads();
        }
}

constexpr int kMaxKeys = GLR_MAX_TOPK, kRadix = 11, kBins = 1 << kRadix;

// The topk largest keys of a row, in `key` in any order: how many there are (fewer where fewer entries are left).  A radix
// selection over the 64-bit keys: 11 bits at a time, the bin in which the topk-th key lies, as far as its ties need.
template <class T>
__device__ int select_keys(const RowVectors<T>& row, int topk, uint64_t* key, int* bins, int* scratch) {
    uint64_t prefix = 0;
    int want = topk, low = 64;                       // bits below `low` are not decided yet; keys share `prefix` above
    bool all = false;
    while (low > 0 && !all) {
        const int bits = min(kRadix, low);
        low -= bits;
        for (int q = threadIdx.x; q < kBins; q += kThreads) bins[q] = 0;
        __syncthreads();
        for (int64_t q = threadIdx.x; q < row.count; q += kThreads) {
            float v[8];
            row.load(q, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint64_t k = key_of(v[e], static_cast<uint32_t>(row.first(q) + e));
                if ((k >> 32) != 0 && (low + bits == 64 || (k >> (low + bits)) == prefix)) atomicAdd(&bins[(k >> low) & ((1 << bits) - 1)], 1);
            }
        }
        __syncthreads();
        // the bin that holds the want-th largest: warp 0 goes through them from the top, 32 at a time
        if (threadIdx.x < 32) {
            const int lane = threadIdx.x;
            int above = 0, bin = -1;
            for (int top = kBins - 32; top >= 0 && bin < 0; top -= 32) {
                const int c = bins[top + 31 - lane];
                int sum = c;
                for (int o = 1; o < 32; o *= 2) { const int y = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += y; }
                const uint32_t past = __ballot_sync(0xffffffffu, above + sum >= want);
                if (past) {
                    const int at = __ffs(past) - 1;
                    bin = top + 31 - at;
                    above += __shfl_sync(0xffffffffu, sum - c, at);
                } else {
                    above += __shfl_sync(0xffffffffu, sum, 31);
                }
            }
            if (lane == 0) { scratch[0] = bin; scratch[1] = above; scratch[2] = bin >= 0 ? bins[bin] : 0; }
        }
        __syncthreads();
        const int bin = scratch[0], above = scratch[1], inside = scratch[2];
        __syncthreads();
        if (bin < 0) { low = 64; prefix = 0; break; }            // fewer than topk entries: all of them (first digit only)
        prefix = prefix << bits | static_cast<uint64_t>(bin);
        want -= above;
        all = inside == want;                        // the whole bin is wanted: its lower bits need no decision
    }
    const uint64_t least = low == 64 ? 1 : prefix << low;
    if (threadIdx.x == 0) scratch[3] = 0;
    __syncthreads();
    for (int64_t q = threadIdx.x; q < row.count; q += kThreads) {
        float v[8];
        row.load(q, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint64_t k = key_of(v[e], static_cast<uint32_t>(row.first(q) + e));
            if ((k >> 32) != 0 && k >= least) {
                const int at = atomicAdd(&scratch[3], 1);
                if (at < topk) key[at] = k;
            }
        }
    }
    __syncthreads();
    return min(scratch[3], topk);
}

template <class T>
__global__ void __launch_bounds__(kThreads) token_logp_kernel(const __grid_constant__ TokenLogp a) {
    chain_begin();
    __shared__ Stat parts[kWarps];
    __shared__ uint64_t key[kMaxKeys];
    __shared__ int bins[kBins];
    __shared__ int scratch[4];
    const int64_t i = blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + i * a.ldz;
    const RowVectors<T> row(z, a.vocab);
    const float c = kLog2e * a.inv_tau;
    Stat t{kLowest, 0.f, 0.f};
    for (int64_t q = threadIdx.x; q < row.count; q += kThreads) {
        float v[8];
        row.load(q, v);
        float m = v[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) m = fmaxf(m, v[e]);
        if (m > t.m) {
            const float d = fmaxf((t.m - m) * c, -1e30f), x = exp2_fast(d);
            t.u = (t.u + t.s * d) * x;
            t.s *= x;
            t.m = m;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = (v[e] - t.m) * c, p = exp2_fast(x);
            t.s += p;
            t.u = fmaf(p, fmaxf(x, -1e30f), t.u);
        }
    }
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const Stat y{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), __shfl_xor_sync(0xffffffffu, t.u, o)};
        t = join(t, y, c);
    }
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = t;
    __syncthreads();
    t = parts[0];
    for (int w = 1; w < kWarps; ++w) t = join(t, parts[w], c);
    const bool some = !(t.s == 0.f);                 // a row with a distribution, or with a NaN
    const float log_s = logf(t.s), lse = t.m * a.inv_tau + log_s;
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[i] = some ? lse : -__int_as_float(0x7f800000);
        if (a.entropy) a.entropy[i] = some ? log_s - t.u * 0.6931471805599453f / t.s : 0.f;
        if (a.logp) {
            const int64_t y = a.tokens.at(i);
            a.logp[i] = some && y >= 0 && y < a.vocab ? (to_f(z[y]) - t.m) * a.inv_tau - log_s : 0.f;
        }
    }
    if (a.topk == 0) return;
    const int n = select_keys(row, a.topk, key, bins, scratch);
    int size = 1;
    while (size < n) size *= 2;
    sort_keys(key, n, size);
    for (int q = threadIdx.x; q < a.topk; q += kThreads) {
        const uint64_t k = q < n ? key[q] : 0;
        const int64_t id = q < n ? static_cast<int64_t>(~static_cast<uint32_t>(k)) : -1;
        if (a.top_logp)
            a.top_logp[i * a.ld_top_logp + q] = q < n ? (logit_of(static_cast<uint32_t>(k >> 32)) - t.m) * a.inv_tau - log_s : -__int_as_float(0x7f800000);
        if (a.top_ids) {
            if (a.ids_wide) static_cast<int64_t*>(a.top_ids)[i * a.ld_top_ids + q] = id;
            else static_cast<int32_t*>(a.top_ids)[i * a.ld_top_ids + q] = static_cast<int32_t>(id);
        }
    }
}

// dz_v = (dlogp (e_token - p_v) - dentropy p_v (log p_v + entropy)) / tau, with log p_v = z_v / tau - lse; the same elements by
// the same thread, so dz may be z.
template <class T>
__global__ void __launch_bounds__(kThreads) token_logp_grad_kernel(const __grid_constant__ TokenLogpGrad a, int parts) {
    chain_begin();
    const int64_t i = blockIdx.x / parts;
    const int part = static_cast<int>(blockIdx.x % parts);
    const T* z = static_cast<const T*>(a.z) + i * a.ldz;
    T* dz = static_cast<T*>(a.dz) + i * a.lddz;
    const RowVectors<T> row(z, a.vocab);
    const int64_t y = a.tokens.p ? a.tokens.at(i) : -1;
    const bool counted = y >= 0 && y < a.vocab;
    const float lse = a.lse[i];
    const bool some = lse != -__int_as_float(0x7f800000);
    const float coef = a.dlogp && counted && some ? a.dlogp[i] * a.inv_tau : 0.f;
    const float bonus = a.dentropy && some ? a.dentropy[i] * a.inv_tau : 0.f, h = bonus != 0.f ? a.entropy[i] : 0.f;
    const float tail = a.inv_tau;
    const bool wide = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z) & 15);
    for (int64_t q = static_cast<int64_t>(part) * kThreads + threadIdx.x; q < row.count; q += static_cast<int64_t>(parts) * kThreads) {
        float v[8];
        row.load(q, v);
        const int64_t j = row.first(q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float lp = v[e] * tail - lse, p = exp2_fast(lp * kLog2e);
            float d = -coef * p;
            if (bonus != 0.f) d -= p != 0.f ? bonus * p * (lp + h) : 0.f;
            if (j + e == y) d += coef;
            v[e] = some && (coef != 0.f || bonus != 0.f) ? d : 0.f;
        }
        T* to = dz + j;
        if (wide && j >= 0 && j + 8 <= a.vocab) {
            store8(to, 8, true, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + e >= 0 && j + e < a.vocab) put(to + e, v[e]);
        }
    }
}

}  // namespace

cudaError_t token_logp(const TokenLogp& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const dim3 grid(static_cast<unsigned>(a.rows));
    return dtype == GLR_BF16 ? launch_chain(token_logp_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a)
                             : launch_chain(token_logp_kernel<float>, grid, kThreads, 0, st, a);
}

cudaError_t token_logp_grad(const TokenLogpGrad& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    // parts of a row of four vectors a thread or more, where there are few rows
    const int64_t most = std::max<int64_t>(1, a.vocab / (8 * 4 * kThreads));
    const int parts = static_cast<int>(std::min(most, std::max<int64_t>(1, 152 * 8 / a.rows)));
    const dim3 grid(static_cast<unsigned>(a.rows * parts));
    return dtype == GLR_BF16 ? launch_chain(token_logp_grad_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, parts)
                             : launch_chain(token_logp_grad_kernel<float>, grid, kThreads, 0, st, a, parts);
}

}  // namespace rows
}  // namespace glr
