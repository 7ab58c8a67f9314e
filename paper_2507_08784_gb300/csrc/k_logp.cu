// Log-probabilities of given tokens with the entropy and the most probable alternatives, and their gradient.
//
// With x_v = (z_v - m) / tau, m the row's maximum, s = sum e^x and u = sum e^x x:
//   lse = m / tau + log s,  logp = x_token - log s,  entropy = log s - u / s  (both terms are of one sign)
// A thread keeps a running maximum and rescales its sums when it grows.  Entries of -infinity add nothing to either sum, and a
// NaN reaches s.  The terms of a round are added up among themselves before they join the thread's sums, which may hold a
// term of 1 (single terms next to it: log p of a token of p = 0.8 among 131071 off by 3e-6 of itself).
//
// The alternatives are ordered by a 64-bit key: the logit as an integer of the same order (-0 as 0, a NaN above all) over the
// complement of its index, so that no two are equal and equal logits go by their index.  They are found in the same pass.  Of the
// CTA's W warps, the lanes of each hold 32 maxima of what they have seen (or several each, of apart vectors); where
// j = ceil(topk / W), the least of the warps' j-th largest maxima has topk elements at or above it, so an element below it is none
// of the alternatives.  This bound is set after the first round, whose elements are still in registers, and raised after
// every doubling; the vectors that hold an element above it (a few hundred of 16384) go to a list in shared memory.  Those
// above the last bound are read again, and their elements put in order by counting or a bitonic sort.
// A list that runs over (many equal logits, every element above those before), a NaN or an infinity, and more alternatives than
// the maxima can bound well are left to a radix selection of the keys, which reads the row again two to six times: for each of
// its digits, one to five, and to collect.
//
// Bound by what it issues beside HBM: 4096 x 131071 bf16 with the entropy and 64 alternatives 234 us (1.07 GB, 4.6 TB/s), 180 without
// alternatives (6.0 TB/s).
//
// A row is a CTA's, or with few rows a cluster's: each CTA takes a part, and ranks its ordered alternatives among those of
// the others, which it reads over distributed shared memory.
#include <algorithm>

#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;

// Exponentials are the hardware's powers of two, within 2^-22 of themselves, of arguments rounded once more for log2(e): what the
// instructions issued allow (see below), and no worse than exp in 32 bits in the sums (of 512 fp32 rows of 32768 both forms'
// log-probabilities are off by 4e-8 of themselves, root mean square).
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

// Two fp32 values in one register pair.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

constexpr float kInf = __builtin_huge_valf();

// Eight neighbouring logits as they lie in memory.
template <class T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void none() { u = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    // those of [from, to) alone
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int from, int to) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t a = 2 * q >= from && 2 * q < to ? h[2 * q] : 0xff80u, b = 2 * q + 1 >= from && 2 * q + 1 < to ? h[2 * q + 1] : 0xff80u;
            w[q] = a | b << 16;
        }
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ float top() const {
        auto h = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
        const __nv_bfloat162 m = __hmax2(__hmax2(h(u.x), h(u.y)), __hmax2(h(u.z), h(u.w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    __device__ __forceinline__ uint64_t pair(int q) const {
        const uint32_t w = q == 0 ? u.x : q == 1 ? u.y : q == 2 ? u.z : u.w;
        return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ __forceinline__ float at(int e) const {
        const uint32_t w = e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w;
        return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void none() { a = b = make_float4(-kInf, -kInf, -kInf, -kInf); }
    __device__ __forceinline__ void load(const float* p, int from, int to) {
        auto at = [&](int e) { return e >= from && e < to ? p[e] : -kInf; };
        a = make_float4(at(0), at(1), at(2), at(3));
        b = make_float4(at(4), at(5), at(6), at(7));
    }
    __device__ __forceinline__ float top() const { return fmaxf(fmaxf(fmaxf(a.x, a.y), fmaxf(a.z, a.w)), fmaxf(fmaxf(b.x, b.y), fmaxf(b.z, b.w))); }
    __device__ __forceinline__ uint64_t pair(int q) const {
        return q == 0 ? pack2(a.x, a.y) : q == 1 ? pack2(a.z, a.w) : q == 2 ? pack2(b.x, b.y) : pack2(b.z, b.w);
    }
    __device__ __forceinline__ float at(int e) const {
        const float4 h = e < 4 ? a : b;
        return (e & 3) == 0 ? h.x : (e & 3) == 1 ? h.y : (e & 3) == 2 ? h.z : h.w;
    }
};

// A row as vectors of eight that begin on 16 bytes, the first one at or before the row's first element: `skip` elements of
// it are not the row's.  A CTA takes the vectors [begin, end).
template <class T>
struct RowVectors {
    const T* base;
    int skip, vocab, begin, end;
    __device__ __forceinline__ RowVectors(const T* z, int v, int part, int parts) : vocab(v) {
        skip = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
        base = z - skip;
        const int count = (skip + v + 7) / 8;
        begin = count * part / parts;
        end = count * (part + 1) / parts;
    }
    __device__ __forceinline__ int first(int q) const { return q * 8 - skip; }     // index of vector q's first element
    // -infinity where there is no element
    __device__ __forceinline__ void load(int q, Eight<T>& v) const {
        const int i = first(q);
        if (q >= end) v.none();
        else if (i >= 0 && i + 8 <= vocab) v.load(base + q * 8);
        else v.load(base + q * 8, i < 0 ? skip : 0, min(8, vocab - i));
    }
    __device__ __forceinline__ void load(int q, float (&v)[8]) const {
        Eight<T> x;
        load(q, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) unpack2(x.pair(e), v[2 * e], v[2 * e + 1]);
    }
};

// The CTA's keys in descending order; the places behind them, up to a power of two, are filled with 0.
template <int NT>
__device__ __noinline__ void sort_keys(uint64_t* key, int n) {
    int size = 1;
    while (size < n) size *= 2;
    for (int q = n + threadIdx.x; q < size; q += NT) key[q] = 0;
    __syncthreads();
    for (int len = 2; len <= size; len *= 2)
        for (int gap = len / 2; gap > 0; gap /= 2) {
            for (int q = threadIdx.x; q < size / 2; q += NT) {
                const int i = 2 * q - (q & (gap - 1)), j = i + gap;
                const uint64_t x = key[i], y = key[j];
                if ((x < y) == ((i & len) == 0)) { key[i] = y; key[j] = x; }
            }
            __syncthreads();
        }
}

constexpr int kMaxKeys = GLR_MAX_TOPK, kRadix = 11, kBins = 1 << kRadix;

// The topk largest keys of the CTA's part of a row, in `key` in any order: how many there are (fewer where fewer entries are
// left).  A radix selection, 11 bits at a time, of the bin in which the topk-th key lies, as far as its ties need.  At least topk
// entries reach `floor`, or it is -infinity, and none is above `most` (in their order): digits are those of
// (order - floor's order, entries behind), whose leading ones differ, and vectors with a maximum below the floor are left out.
// (With the digits of the keys themselves thousands of atomics met in a few bins: 1024 rows of 131072 equal logits 1.35 ms, now
// 0.45.)  Nearly every warp has a lane above the floor in every vector, so a pass costs a warp all its entries: 4096 x 131072
// bf16 with 1024 alternatives take 3.1 ms.
template <class T, int NT>
__device__ __noinline__ int select_keys(const RowVectors<T>& row, int topk, float floor, uint32_t most, uint64_t* key, int* bins, int* scratch) {
    const uint32_t least_order = max(1u, order_of(floor));
    const int index_bits = 32 - __clz(row.vocab);
    const auto digits_of = [&](uint32_t order, int index) {
        return static_cast<uint64_t>(order - least_order) << index_bits | static_cast<uint32_t>(row.vocab - 1 - index);
    };
    // every entry of the vectors that hold one at or above the floor; four loads ahead
    const auto visit = [&](const auto& take) {
        for (int q0 = row.begin; q0 < row.end; q0 += 4 * NT) {
            Eight<T> v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) row.load(q0 + u * NT + threadIdx.x, v[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (v[u].top() < floor) continue;    // (false of eight NaNs, whose maximum is one)
                for (int e = 0; e < 8; ++e) {
                    const float x = v[u].at(e);
                    const int index = row.first(q0 + u * NT + threadIdx.x) + e;
                    if (order_of(x) >= least_order) take(x, index, digits_of(order_of(x), index));
                }
            }
        }
    };
    uint64_t prefix = 0;
    int want = topk, low = 64 - __clzll(digits_of(max(most, least_order), 0));     // bits below `low` are not decided yet
    bool every = false;
    while (low > 0) {
        const int bits = min(kRadix, low);
        low -= bits;
        for (int q = threadIdx.x; q < kBins; q += NT) bins[q] = 0;
        __syncthreads();
        visit([&](float, int, uint64_t d) {
            if (d >> (low + bits) == prefix) atomicAdd(&bins[(d >> low) & ((1 << bits) - 1)], 1);
        });
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
        if (bin < 0) { every = true; break; }        // fewer than topk entries: all of them (first digit only)
        prefix = prefix << bits | static_cast<uint64_t>(bin);
        want -= above;
        // the bin's least entry is a better floor (not where a NaN or an infinity may be it: all vectors are looked at then)
        if (most != 0xffffffffu) floor = fmaxf(floor, logit_of(least_order + static_cast<uint32_t>((prefix << low) >> index_bits)));
        if (inside == want) break;                   // the whole bin is wanted: its lower bits need no decision
    }
    const uint64_t least = every ? 0 : prefix << low;
    if (threadIdx.x == 0) scratch[3] = 0;
    __syncthreads();
    visit([&](float x, int index, uint64_t d) {
        if (d < least) return;
        const int at = atomicAdd(&scratch[3], 1);
        if (at < topk) key[at] = key_of(x, static_cast<uint32_t>(index));
    });
    __syncthreads();
    return min(scratch[3], topk);
}

// The j-th largest of the lanes' values.
__device__ __forceinline__ float lanes_largest(float v, int j) {
    uint32_t o = order_of(v), most = 0;
    for (int left = j; left > 0;) {
        most = __reduce_max_sync(0xffffffffu, o);
        left -= __popc(__ballot_sync(0xffffffffu, o == most));       // equal ones at once
        if (o == most) o = 0;
    }
    return most == 0 ? kLowest : fmaxf(logit_of(most), kLowest);
}
// A value that at least j of the lanes' n values each reach, j <= 32 n: at most sixteen bisections between the least and the
// largest of them, as integers of the same order (1 is that of no logit, and below all of them).
template <int N>
__device__ __noinline__ float lanes_many(const float (&v)[N], int j) {
    uint32_t o[N], lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int q = 0; q < N; ++q) { o[q] = order_of(v[q]); lo = min(lo, o[q]); hi = max(hi, o[q]); }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    for (int it = 0; it < 16 && hi - lo > 1; ++it) {
        const uint32_t mid = lo + (hi - lo) / 2;
        int n = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) n += __popc(__ballot_sync(0xffffffffu, o[q] >= mid));
        if (n >= j) lo = mid; else hi = mid;
        if (n == j) break;                           // (8192 x 8192 bf16, 128 alternatives 146 us without, 142 so)
    }
    return fmaxf(logit_of(lo), kLowest);
}

// The order of an entry's maximum, of which it has the upper half: no less than the upper half of the maximum's own order.
__device__ __forceinline__ uint32_t entry_order(uint32_t entry) { return order_of(__uint_as_float(entry & 0xffff0000u)); }

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    return a;
}
__device__ __forceinline__ uint64_t peer_key(const uint64_t* p, uint32_t rank) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer_addr(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float peer_float(const float* p, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer_addr(p, rank)) : "memory");
    return v;
}

// Vectors a thread loads at once (their running maxima are kept apart), and how many alternatives the list is used for: with one
// maximum a lane, and with all.
template <class T> constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;
constexpr int kCounted = 256;
template <class T, int NT> constexpr int kFew = NT / 2;
template <class T, int NT> constexpr int kListed = NT * kAhead<T> * 3 / 8;
// Entropy and alternatives or not: both cost arithmetic in every element.
template <class T, bool ENT, bool TOP, int NT>
__global__ void __launch_bounds__(NT, 1280 / NT) token_logp_kernel(const __grid_constant__ TokenLogp a, int parts) {
    chain_begin();
    constexpr int W = NT / 32, kWarpList = kMaxKeys * 2 / W;
    __shared__ Stat stats[W + 1];
    __shared__ float bounds[W];
    __shared__ int scratch[4];
    // Each warp's vectors that hold an element above the bound, with the upper half of their maximum; the ordered keys in the
    // end.  (16 KiB in all: the loads' lines in flight need the rest of the SM's memory, with 40 KiB a CTA 4096 rows took 30 us more.)
    __shared__ __align__(16) uint64_t ordered[TOP ? kMaxKeys : 1];
    uint32_t* list = reinterpret_cast<uint32_t*>(ordered);
    __shared__ uint64_t thin[TOP ? kMaxKeys : 1];    // the elements above the last bound (the radix selection's bins)
    __shared__ int over, thin_count;
    static_assert(kBins * sizeof(int) <= kMaxKeys * sizeof(uint64_t), "");
    const uint32_t part = parts > 1 ? cluster_rank() : 0;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float c = kLog2e * a.inv_tau;
    const uint64_t c2 = pack2(c, c);
    const bool listed = TOP && a.topk <= kListed<T, NT>, few = a.topk <= kFew<T, NT>;
    const int mine = (a.topk + W - 1) / W;
    constexpr int A = kAhead<T>;
    const int64_t i = blockIdx.x / parts;
    const T* z = static_cast<const T*>(a.z) + i * a.ldz;
    const RowVectors<T> row(z, static_cast<int>(a.vocab), static_cast<int>(part), parts);
    if (TOP) {
        if (threadIdx.x == 0) { over = 0; thin_count = 0; }
        __syncthreads();
    }
    Stat t{kLowest, 0.f, 0.f};
    float bound = kLowest, most[A];
#pragma unroll
    for (int y = 0; y < A; ++y) most[y] = kLowest;
    int round = 0, due = 0, entries = 0;
    const uint32_t before = (1u << lane) - 1;
    uint32_t* mine_list = list + warp * kWarpList;
    // the warp's entries that a new bound leaves move up
    const auto thin_out = [&](float b) {
        const uint32_t least = order_of(b) & 0xffff0000u;
        int kept = 0;
        __syncwarp();
        for (int q = 0; q < entries; q += 32) {
            const uint32_t entry = q + lane < entries ? mine_list[q + lane] : 0;
            const uint32_t some = __ballot_sync(0xffffffffu, q + lane < entries && entry_order(entry) >= least);
            if (some >> lane & 1) mine_list[kept + __popc(some & before)] = entry;
            kept += __popc(some);
            __syncwarp();
        }
        entries = kept;
    };
    for (int q0 = row.begin; q0 < row.end; q0 += A * NT, ++round) {
        Eight<T> v[A];
        float top[A];
        if (q0 > row.begin && q0 + A * NT < row.end) {       // whole vectors all of them
            const T* p = row.base + (q0 + static_cast<int>(threadIdx.x)) * 8;
#pragma unroll
            for (int y = 0; y < A; ++y) v[y].load(p + y * NT * 8);
        } else {
#pragma unroll
            for (int y = 0; y < A; ++y) row.load(q0 + y * NT + threadIdx.x, v[y]);
        }
        float m_round = -kInf;
#pragma unroll
        for (int y = 0; y < A; ++y) { top[y] = v[y].top(); m_round = fmaxf(m_round, top[y]); }
        if (TOP && !few) {
#pragma unroll
            for (int y = 0; y < A; ++y) most[y] = fmaxf(most[y], top[y]);
        }
        const float m = fmaxf(t.m, m_round);
        if (m > t.m) {
            const float d = fmaxf((t.m - m) * c, -1e30f), x = exp2_fast(d);
            t.u = (t.u + t.s * d) * x;
            t.s *= x;
            t.m = m;
        }
        const uint64_t neg = pack2(-t.m, -t.m);
        uint64_t s2 = 0, u2 = 0;                     // two sums of 0.f
#pragma unroll
        for (int y = 0; y < A; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x0, x1;
                unpack2(mul2(add2(v[y].pair(e), neg), c2), x0, x1);
                const uint64_t p = pack2(exp2_fast(x0), exp2_fast(x1));
                s2 = add2(s2, p);
                // beyond 2^-126 the exponential is 0; -infinity is no factor for it
                if (ENT) u2 = fma2(p, pack2(fmaxf(x0, -200.f), fmaxf(x1, -200.f)), u2);
            }
        float s0, s1;
        unpack2(s2, s0, s1);
        t.s += s0 + s1;
        if (ENT) { unpack2(u2, s0, s1); t.u += s0 + s1; }
        if (listed) {
            // after 1, 2, 4, ... rounds, but the last
            if (round == due && (round == 0 || q0 + A * NT < row.end)) {
                due = 2 * due + 1;
                const float least = few ? lanes_largest(t.m, mine) : lanes_many(most, mine);
                if (lane == 0) bounds[warp] = least;
                __syncthreads();                     // a warp far behind would keep the bound down for all
                float b = bounds[lane & (W - 1)];       // (a later one is a bound too)
#pragma unroll
                for (int o = 1; o < W; o *= 2) b = fminf(b, __shfl_xor_sync(0xffffffffu, b, o));
                bound = fmaxf(bound, b);
                if (entries > kWarpList / 4 && entries <= kWarpList) thin_out(bound);
            }
            if (__any_sync(0xffffffffu, m_round >= bound)) {
                const uint32_t place = static_cast<uint32_t>(round * A * 32 + lane);
#pragma unroll
                for (int y = 0; y < A; ++y) {
                    const uint32_t some = __ballot_sync(0xffffffffu, top[y] >= bound);
                    if (some == 0) continue;
                    const int at = entries + __popc(some & before);
                    if (top[y] >= bound && at < kWarpList) mine_list[at] = (__float_as_uint(top[y]) & 0xffff0000u) | (place + y * 32);
                    entries += __popc(some);
                }
            }
        }
    }
    // a part of one round: its first bound is the last one (16384 x 2048 bf16, 64 alternatives 126 us with both, 103 with one)
    const bool current = listed && round == 1;
    if (TOP && !current) {
        const float least = few ? lanes_largest(t.m, mine) : mine <= 32 * A ? lanes_many(most, mine) : kLowest;
        if (lane == 0) bounds[warp] = least;
    }
    if (TOP && lane == 0 && entries > kWarpList) atomicAdd(&over, 1);
    // the CTA's statistics, then the row's
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const Stat y{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), __shfl_xor_sync(0xffffffffu, t.u, o)};
        t = join(t, y, c);
    }
    if (lane == 0) stats[warp] = t;
    __syncthreads();
    t = stats[0];
    for (int w = 1; w < W; ++w) t = join(t, stats[w], c);
    int n = 0;
    if (TOP && row.begin < row.end) {
        bool done = false;
        float b = bounds[0];
#pragma unroll
        for (int w = 1; w < W; ++w) b = fminf(b, bounds[w]);
        const bool ordinary = t.s < kInf;            // no NaN and no infinity in this part
        if (listed && over == 0 && ordinary) {
            if (!current) thin_out(b);               // first, so that most are read again at once
            for (int q = lane; q < entries; q += 32) {
                const uint32_t entry = mine_list[q];
                const int at = row.begin + static_cast<int>(entry >> 5 & 0x7ffu) * NT + warp * 32 + static_cast<int>(entry & 31);
                Eight<T> v;
                row.load(at, v);
                for (int e = 0; e < 8; ++e) {
                    const float x = v.at(e);
                    if (!(x >= b)) continue;
                    const int to = atomicAdd(&thin_count, 1);
                    if (to < kMaxKeys) thin[to] = key_of(x, static_cast<uint32_t>(row.first(at) + e));
                }
            }
            __syncthreads();
            n = thin_count;
            done = n <= kMaxKeys;
            if (n <= kCounted) {
                for (int q = threadIdx.x; q < n; q += NT) {
                    const uint64_t k = thin[q];
                    int above = 0;
                    for (int r = 0; r < n; ++r) above += thin[r] > k;
                    ordered[above] = k;
                }
                __syncthreads();
            } else if (done) {
                for (int q = threadIdx.x; q < n; q += NT) ordered[q] = thin[q];
                sort_keys<NT>(ordered, n);
            }
        }
        if (!done) {
            __syncthreads();
            n = select_keys<T, NT>(row, a.topk, ordinary ? b : -kInf, ordinary ? order_of(t.m) : 0xffffffffu, ordered, reinterpret_cast<int*>(thin), scratch);
            sort_keys<NT>(ordered, n);
        }
        n = min(n, a.topk);
    }
    if (parts > 1) {
        if (threadIdx.x == 0) { stats[W] = t; scratch[3] = n; }
        cluster_sync();
        // a CTA's statistics a lane, joined in the same order everywhere
        t = Stat{kLowest, 0.f, 0.f};
        if (lane < parts) {
            const float* f = &stats[W].m;
            t = Stat{peer_float(f, lane), peer_float(f + 1, lane), peer_float(f + 2, lane)};
        }
        for (int o = 1; o < parts; o *= 2) {
            const Stat y{__shfl_down_sync(0xffffffffu, t.m, o), __shfl_down_sync(0xffffffffu, t.s, o), __shfl_down_sync(0xffffffffu, t.u, o)};
            t = join(t, y, c);
        }
        t = Stat{__shfl_sync(0xffffffffu, t.m, 0), __shfl_sync(0xffffffffu, t.s, 0), __shfl_sync(0xffffffffu, t.u, 0)};
    }
    const bool some = !(t.s == 0.f);                 // a row with a distribution, or with a NaN
    const float log_s = logf(t.s);
    if (threadIdx.x == 0 && part == 0) {
        if (a.lse) a.lse[i] = some ? t.m * a.inv_tau + log_s : -kInf;
        if (ENT) a.entropy[i] = some ? log_s - t.u * 0.6931471805599453f / t.s : 0.f;
        if (a.logp) {
            const int64_t y = a.tokens.at(i);
            a.logp[i] = some && y >= 0 && y < a.vocab ? (to_f(z[y]) - t.m) * a.inv_tau - log_s : 0.f;
        }
    }
    if (!TOP) {
        if (parts > 1) cluster_sync();
        return;
    }
    const auto write = [&](int at, uint64_t k) {           // k = 0: none left
        if (a.top_logp) a.top_logp[i * a.ld_top_logp + at] = k ? (logit_of(static_cast<uint32_t>(k >> 32)) - t.m) * a.inv_tau - log_s : -kInf;
        if (a.top_ids) {
            const int64_t id = k ? static_cast<int64_t>(~static_cast<uint32_t>(k)) : -1;
            if (a.ids_wide) static_cast<int64_t*>(a.top_ids)[i * a.ld_top_ids + at] = id;
            else static_cast<int32_t*>(a.top_ids)[i * a.ld_top_ids + at] = static_cast<int32_t>(id);
        }
    };
    if (parts == 1) {
        for (int q = threadIdx.x; q < a.topk; q += NT) write(q, q < n ? ordered[q] : 0);
        return;
    }
    // each CTA's keys go where they rank among all of them: a thread counts those of one peer above one key
    const auto keys_of = [&](uint32_t rank) { return __float_as_int(peer_float(reinterpret_cast<const float*>(scratch + 3), rank)); };
    const int total = __reduce_add_sync(0xffffffffu, lane < parts ? keys_of(lane) : 0);
    int* above = reinterpret_cast<int*>(thin);
    for (int q = threadIdx.x; q < n; q += NT) above[q] = q;
    __syncthreads();
    for (int q = threadIdx.x; q < n * (parts - 1); q += NT) {
        const int own = q % n;
        const uint32_t peer = (part + 1 + q / n) % parts;
        const uint64_t k = ordered[own];
        int lo = 0, hi = keys_of(peer);
        while (lo < hi) { const int mid = (lo + hi) >> 1; if (peer_key(ordered + mid, peer) > k) lo = mid + 1; else hi = mid; }
        if (lo) atomicAdd(&above[own], lo);
    }
    __syncthreads();
    for (int q = threadIdx.x; q < n; q += NT)
        if (above[q] < a.topk) write(above[q], ordered[q]);
    if (part == 0)
        for (int q = total + threadIdx.x; q < a.topk; q += NT) write(q, 0);
    cluster_sync();
}

// dz_v = (dlogp (e_token - p_v) - dentropy p_v (log p_v + entropy)) / tau, with log p_v = z_v / tau - lse; the same elements by
// the same thread, so dz may be z.  Bound by HBM: 6000 x 65536 bf16 with both terms 231 us, 6.8 TB/s
// (one vector's load at a time 293).
template <class T> constexpr int kGradAhead = sizeof(T) == 2 ? 4 : 2;

// lse is one fp32 number, off by up to |lse| 2^-24, and z / tau by as much: up to 64 that leaves every p within 2^-16 of itself.
// Beyond (logits far from zero, rows of the type's lowest value, an m / tau that leaves the range) the row's maximum and sum
// are formed again, and log p_v = (z_v - m) / tau - log s (6000 x 65536 bf16, all rows such: 378 us; one of 131072 18, in place 30).
constexpr float kFar = 64.f;

// The CTA's Stat (without u) of a whole row.  Not inlined: few rows need it, and its registers would be every row's.
template <class T>
__device__ __noinline__ Stat row_stat(const T* z, int vocab, float c) {
    __shared__ Stat stats[kThreads / 32];
    constexpr int A = kGradAhead<T>;
    const RowVectors<T> row(z, vocab, 0, 1);
    Stat t{kLowest, 0.f, 0.f};
    for (int q0 = row.begin; q0 < row.end; q0 += A * kThreads) {
        Eight<T> x[A];
        float m = t.m, s = 0.f;
#pragma unroll
        for (int u = 0; u < A; ++u) { row.load(q0 + u * kThreads + threadIdx.x, x[u]); m = fmaxf(m, x[u].top()); }
#pragma unroll
        for (int u = 0; u < A; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += exp2_fast((x[u].at(e) - m) * c);
        t.s = fmaf(t.s, exp2_fast((t.m - m) * c), s);
        t.m = m;
    }
#pragma unroll
    for (int o = 1; o < 32; o *= 2) t = join(t, Stat{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), 0.f}, c);
    if ((threadIdx.x & 31) == 0) stats[threadIdx.x >> 5] = t;
    __syncthreads();
    t = stats[0];
    for (int w = 1; w < kThreads / 32; ++w) t = join(t, stats[w], c);
    return t;
}

template <class T, bool ENT>
__global__ void __launch_bounds__(kThreads) token_logp_grad_kernel(const __grid_constant__ TokenLogpGrad a, int parts) {
    chain_begin();
    constexpr int A = kGradAhead<T>;
    const int64_t i = blockIdx.x / parts;
    const int part = static_cast<int>(blockIdx.x % parts);
    const T* z = static_cast<const T*>(a.z) + i * a.ldz;
    T* dz = static_cast<T*>(a.dz) + i * a.lddz;
    RowVectors<T> row(z, static_cast<int>(a.vocab), part, parts);
    const int64_t y64 = a.tokens.p ? a.tokens.at(i) : -1;
    const int y = y64 >= 0 && y64 < a.vocab ? static_cast<int>(y64) : -8;
    float lse = a.lse[i], m = 0.f;
    float coef = a.dlogp && y >= 0 ? a.dlogp[i] * a.inv_tau : 0.f;
    float bonus = ENT ? a.dentropy[i] * a.inv_tau : 0.f;
    bool read = coef != 0.f || bonus != 0.f;         // (a NaN among them too)
    const bool far = read && fabsf(lse) > kFar;      // the same for all CTAs of a row
    if (far) {
        if (a.dz == a.z) {                           // one CTA for all of it: another would read what it has written
            if (part) return;
            row = RowVectors<T>(z, static_cast<int>(a.vocab), 0, 1);
        }
        const Stat t = row_stat(z, static_cast<int>(a.vocab), kLog2e * a.inv_tau);
        m = t.m;
        lse = logf(t.s);
        if (t.s == 0.f) { read = false; coef = bonus = 0.f; }        // no distribution
    }
    // the factor of p: -coef - bonus (log p + entropy)
    const float base = -(bonus != 0.f ? fmaf(bonus, a.entropy[i], coef) : coef);
    const bool wide = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z) & 15);
    for (int q0 = row.begin; q0 < row.end; q0 += A * kThreads) {
        Eight<T> x[A];
        const bool inside = q0 > row.begin && q0 + A * kThreads < row.end;   // whole vectors all of them
        if (!read) {
#pragma unroll
            for (int u = 0; u < A; ++u) x[u].none();
        } else if (inside) {
            const T* p = row.base + (q0 + static_cast<int>(threadIdx.x)) * 8;
#pragma unroll
            for (int u = 0; u < A; ++u) x[u].load(p + u * kThreads * 8);
        } else {
#pragma unroll
            for (int u = 0; u < A; ++u) row.load(q0 + u * kThreads + threadIdx.x, x[u]);
        }
#pragma unroll
        for (int u = 0; u < A; ++u) {
            const int q = q0 + u * kThreads + threadIdx.x, j = row.first(q);
            if (q >= row.end) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) unpack2(x[u].pair(e), v[2 * e], v[2 * e + 1]);
            if (far) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] -= m;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float lp = fmaf(v[e], a.inv_tau, -lse), p = exp2_fast(lp * kLog2e);
                // (below 2^-126 p is 0, and a log p of -infinity no factor for it)
                v[e] = !read ? 0.f : ENT ? p * fmaf(-bonus, fmaxf(lp, -200.f), base) : p * base;
            }
            if (y >= j && y < j + 8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += j + e == y ? coef : 0.f;
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
}

template <class T, int NT>
auto logp_kernel_of(const TokenLogp& a) {
    return a.entropy ? (a.topk ? token_logp_kernel<T, true, true, NT> : token_logp_kernel<T, true, false, NT>)
                     : (a.topk ? token_logp_kernel<T, false, true, NT> : token_logp_kernel<T, false, false, NT>);
}
template <class T>
auto logp_kernel(const TokenLogp& a, int threads) {
    return threads == 64 ? logp_kernel_of<T, 64>(a) : threads == 128 ? logp_kernel_of<T, 128>(a) : logp_kernel_of<T, 256>(a);
}

}  // namespace

cudaError_t token_logp(const TokenLogp& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    // CTAs a row: a cluster where the rows leave SMs idle, each CTA with 4096 logits at least
    int parts = 1;
    while (parts < 8 && a.rows * parts * 2 <= 2 * 152 && a.vocab >= parts * 2 * 4096) parts *= 2;
    // Threads a CTA: smaller ones are more in turn at a row's end (4096 x 131071 bf16, 64 alternatives: 246 us with 128, 262 with 256,
    // 331 with 64; 16384 x 5003 without alternatives 66 with 128, 51 with 64), but bound fewer alternatives, and share fewer keys'
    // ordering in a cluster (one row of 32768, 64 alternatives: 13 with 128, 9 with 256).
    const auto listed = [&](int threads) { return threads * (dtype == GLR_BF16 ? kAhead<__nv_bfloat16> : kAhead<float>) * 3 / 8; };
    int threads = a.vocab <= (a.topk ? 2048 : 8192) && a.topk <= listed(64) ? 64 : 128;
    if (threads == 128 && (a.topk > std::min(128, listed(128)) || (parts > 1 && a.topk > 32))) threads = 256;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = parts; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(a.rows * parts)); cfg.blockDim = threads; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = parts > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, dtype == GLR_BF16 ? logp_kernel<__nv_bfloat16>(a, threads) : logp_kernel<float>(a, threads), a, parts);
}

cudaError_t token_logp_grad(const TokenLogpGrad& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    // parts of a row of four vectors a thread or more, where there are few rows
    const int64_t most = std::max<int64_t>(1, a.vocab / (8 * 4 * kThreads));
    const int parts = static_cast<int>(std::min(most, std::max<int64_t>(1, 152 * 8 / a.rows)));
    const dim3 grid(static_cast<unsigned>(a.rows * parts));
    using H = __nv_bfloat16;
    return launch_chain(dtype == GLR_BF16 ? (a.dentropy ? token_logp_grad_kernel<H, true> : token_logp_grad_kernel<H, false>)
                                          : (a.dentropy ? token_logp_grad_kernel<float, true> : token_logp_grad_kernel<float, false>),
                        grid, kThreads, 0, st, a, parts);
}

}  // namespace rows
}  // namespace glr
