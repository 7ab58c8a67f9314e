// Losses on logits with their gradients: distillation from a teacher's top logits, the clipped policy
// loss, and the log-probabilities, pairs and gradient of the preference loss.
//
// A row's statistics are the running maximum m and sums s = sum exp((z - m) / tau) of a softmax;
// log p_v = (z_v - m) / tau - log s and p_v = exp((z_v - m) / tau) / s.  Everything is formed from
// z - m, so logits of the type's lowest value and of -infinity need no special case: m is taken as 0
// where every logit is -infinity (then s = 0: the row leaves no distribution), and a NaN reaches s.
//
// The rows kernel reads a row once and writes its gradient once.  A row, or with a cluster of C CTAs a
// C-th of it, lies in a slot of shared memory: filled by a bulk copy while earlier rows are worked on,
// reduced by all warps, overwritten by its own gradient and written back by a bulk copy.  The
// CTAs of a cluster exchange (m, s) over distributed shared memory.  So it is bound by HBM as long as a
// row's arithmetic (two exponentials and about eight instructions a logit) is shorter than its copies.
#include <math_constants.h>

#include <algorithm>

#include "glr_loss.cuh"
#include "glr_ptx.cuh"

namespace glr {
namespace loss {

namespace {

using tc::mbar_expect_tx;
using tc::mbar_init;
using tc::smem_u32;

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float load(const float* p) { return *p; }
__device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

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
__device__ __forceinline__ uint64_t exp2_2(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    return pack2(exp2_fast(a), exp2_fast(b));
}

// Sixteen bytes of logits as pairs, and back.
template <class T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int kElems = 8;
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __forceinline__ void get(const uint4& u, uint64_t (&v)[4]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = pack2(__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u));
    }
    static __device__ __forceinline__ float top(const uint4& u) {
        auto h = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
        const __nv_bfloat162 m = __hmax2(__hmax2(h(u.x), h(u.y)), __hmax2(h(u.z), h(u.w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ uint4 put(const uint64_t (&v)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float a, b;
            unpack2(v[q], a, b);
            const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
            w[q] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec<float> {
    static constexpr int kElems = 4;
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    static __device__ __forceinline__ void get(const uint4& u, uint64_t (&v)[2]) {
        v[0] = pack2(__uint_as_float(u.x), __uint_as_float(u.y));
        v[1] = pack2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ float top(const uint4& u) {
        return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
    }
    static __device__ __forceinline__ uint4 put(const uint64_t (&v)[2]) {
        float a, b, c, d;
        unpack2(v[0], a, b);
        unpack2(v[1], c, d);
        return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
    }
};

// exp2((a - m) c) for a <= m, with -infinity against -infinity counted as 1 (its sum is 0)
__device__ __forceinline__ float shrink(float a, float m, float c) {
    return a == -CUDART_INF_F ? 1.f : exp2_fast((a - m) * c);
}
// Maximum, and sums of exp at two temperatures (s1: temperature 1, for a hard term beside tau != 1).
struct Stat { float m, s, s1; };
// Teacher: maximum, sums of e = exp((a - m) / tau) and of e (a - m).
struct Top { float m, s, a; };
__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}
// The merge of a warp's lanes, in a fixed order, to all of them: one maximum, every lane's sums taken to it,
// and their sum.  A NaN does not show in a maximum; it stays in the sums.
__device__ __forceinline__ Stat warp_merge(Stat x, float c, bool two) {
    Stat r;
    r.m = warp_max(x.m);
    r.s = warp_sum(x.s * shrink(x.m, r.m, c));
    r.s1 = two ? warp_sum(x.s1 * shrink(x.m, r.m, kLog2e)) : 0.f;
    return r;
}
__device__ __forceinline__ Top warp_merge(Top x, float c) {
    Top r;
    r.m = warp_max(x.m);
    const float f = shrink(x.m, r.m, c);
    r.s = warp_sum(x.s * f);
    r.a = warp_sum(x.s == 0.f ? 0.f : (x.a + x.s * (x.m - r.m)) * f);
    return r;
}

constexpr int kMaxWarps = 16;
constexpr int kMaxSlots = 4;
constexpr int kMaxCluster = 8;
constexpr int kEntries = 2;                 // teacher entries a thread: topk <= 2 x threads
constexpr int kHeld = 8;                    // 16-byte vectors of a slot whose exponentials a thread keeps in registers

__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Bounded wait.  One that gives up raises the CTA's abort flag and counts; from then on every wait of the
// CTA returns at once, so that its threads still meet at their barriers and leave together.
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile int* abort, int* err) {
    for (int it = 0; it < 16000000; ++it) {
        if (try_wait(bar, parity)) return;
        if (it >= 64) {
            if (*abort) return;
            __nanosleep(64);
        }
    }
    if (atomicExch(const_cast<int*>(abort), 1) == 0) atomicAdd(err, 1);
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// What a row needs beside its logits.  It is loaded a row ahead and looked at only then: an index stays as its
// two words, and nothing is compared or converted on the way, which would wait for memory.
struct Word { int32_t lo, hi; };
__device__ __forceinline__ Word word_at(const Index& x, int64_t i) {
    if (x.wide) {
        const int2 v = static_cast<const int2*>(x.p)[i];
        return {v.x, v.y};
    }
    return {static_cast<const int32_t*>(x.p)[i], 0};
}
// The index if it lies in [0, vocab), else -1.
__device__ __forceinline__ int32_t index_of(const Word& w, int wide, int vocab) {
    return (!wide || w.hi == 0) && w.lo >= 0 && w.lo < vocab ? w.lo : -1;
}
struct Side {
    float w, adv, old, ref;
    Word tok;
};
template <int K>
__device__ __forceinline__ Side side_at(const RowArgs& a, int64_t row, bool full) {
    Side s{};
    s.w = K == kLogProb ? 1.f : a.weight ? a.weight[row] : a.share;
    s.tok = {-1, 0};
    if (K != kDistill) s.tok = word_at(a.tokens, row);
    else if (a.labels.p && full) s.tok = word_at(a.labels, row);
    if (K == kPolicy && full) {
        s.adv = a.advantage[row];
        s.old = a.old_logp[row];
        if (a.ref_logp) s.ref = a.ref_logp[row];
    }
    return s;
}
template <int K>
__device__ __forceinline__ int32_t token_of(const RowArgs& a, const Side& s) {
    return index_of(s.tok, K == kDistill ? a.labels.wide : a.tokens.wide, static_cast<int>(a.vocab));
}
template <int K>
__device__ __forceinline__ bool is_live(const RowArgs& a, const Side& s) {
    return s.w != 0.f && (K == kDistill || token_of<K>(a, s) >= 0);
}
// The 16-byte vectors of a row between its unaligned ends, and this CTA's share of them.
struct Span {
    int head, tail;                          // elements before and after the vectors
    int v0, v1;                              // vectors [v0, v1) are this CTA's
    int elems;                               // in all the vectors
};
template <class T>
__device__ __forceinline__ Span span_of(const T* z, int vocab, int rank, int csize) {
    constexpr int E = Vec<T>::kElems;
    Span s;
    s.head = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(T));
    s.head = s.head < vocab ? s.head : vocab;
    const int n = (vocab - s.head) / E, per = (n + csize - 1) / csize;
    s.elems = n * E;
    s.tail = vocab - s.head - s.elems;
    s.v0 = min(rank * per, n);
    s.v1 = min(s.v0 + per, n);
    return s;
}

constexpr int64_t kSlotMax = kMaxWarps * 32 * kHeld * 16;    // of a row a CTA: 64 KiB, three slots fit
constexpr int64_t kRingMax = 208 * 1024;

// HELD: a slot has at most kHeld vectors a thread, and the exponentials of the statistics stay in registers
// for the gradient; else (rows of more than eight such slots) they are formed again.
template <int K, class T, bool HELD>
__global__ void __launch_bounds__(kMaxWarps * 32) rows_kernel(const __grid_constant__ RowArgs a) {
    chain_begin();
    constexpr int E = Vec<T>::kElems, P = E / 2;
    constexpr int kKeep = HELD && K != kLogProb ? kHeld : 1;
    extern __shared__ __align__(128) uint8_t slots[];
    __shared__ __align__(8) uint64_t full_bar[kMaxSlots], x_bar[2];
    // by the row's parity: a warp may be a row ahead of one that still reads
    __shared__ Stat stat_s[2][kMaxWarps], cluster_s[2][kMaxCluster];
    __shared__ Top top_s[2][K == kDistill ? kMaxWarps : 1];
    __shared__ float zq_s[K == kDistill ? kMaxWarps : 1];
    __shared__ int32_t id_s[K == kDistill ? GLR_MAX_TOPK + 1 : 1];
    __shared__ float q_s[K == kDistill ? GLR_MAX_TOPK + 1 : 1];
    __shared__ int32_t edge_s[16];
    __shared__ int abort_flag;
    const int nt = blockDim.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nw = nt >> 5;
    const int C = a.cluster, S = a.slots, V = static_cast<int>(a.vocab);
    uint32_t rank = 0;
    if (C > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int64_t first = blockIdx.x / C, step = gridDim.x / C;
    volatile int* abort = &abort_flag;
    if (tid == 0) {
        abort_flag = 0;
        for (int q = 0; q < S; ++q) mbar_init(smem_u32(&full_bar[q]), 1);
        mbar_init(smem_u32(&x_bar[0]), C);
        mbar_init(smem_u32(&x_bar[1]), C);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (C > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    const bool grad = K != kLogProb && a.dz != nullptr;

    // Thread 0 fills the slots, and writes them back once every thread is done with a row.
    int64_t next = first;
    Side ask{};                                       // the next row to fill: whether it is read
    int fs = 0;
    uint32_t filled = 0, fill_par = 0;                // per slot (bit q): filled at all, parity of the last fill
    auto fill = [&]() {
        if (next >= a.rows) return;
        const T* z = static_cast<const T*>(a.z) + next * a.ldz;
        const Span sp = span_of(z, V, rank, C);
        const uint32_t bytes = is_live<K>(a, ask) ? static_cast<uint32_t>(sp.v1 - sp.v0) * 16u : 0u;
        const uint32_t bar = smem_u32(&full_bar[fs]);
        mbar_expect_tx(bar, bytes);
        if (bytes)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_u32(slots + static_cast<size_t>(fs) * a.slot_bytes)), "l"(z + sp.head + static_cast<int64_t>(sp.v0) * E),
                         "r"(bytes), "r"(bar) : "memory");
        fill_par = filled >> fs & 1u ? fill_par ^ 1u << fs : fill_par;
        filled |= 1u << fs;
        if (++fs == S) fs = 0;
        next += step;
        if (next < a.rows) ask = side_at<K>(a, next, false);
    };
    // with a gradient the slot of the row before is filled while this one's is written back (S = 1: its own)
    if (tid == 0) {
        if (first < a.rows) ask = side_at<K>(a, first, false);
        for (int q = 0; q < (grad && S > 1 ? S - 1 : S); ++q) fill();
    }

    const float c = a.inv_tau * kLog2e;
    const bool two = K == kDistill && a.labels.p && a.hard != 0.f && a.inv_tau != 1.f;
    const uint64_t c2 = pack2(c, c), l2 = pack2(kLog2e, kLog2e);
    int s = 0, par = 0;
    uint32_t use = 0, xuse = 0;
    Side side{};
    Word id[kEntries];
    float av[kEntries];                                // bf16 teacher logits as their bits
    T edge;
    // Row data of `row`, ahead of their use: everything but what lies in the slot.
    auto ahead = [&](int64_t row) {
        side = side_at<K>(a, row, true);
        if (K == kDistill) {
#pragma unroll
            for (int u = 0; u < kEntries; ++u) {
                const int k = tid + u * nt;
                if (k < a.topk) {
                    id[u] = word_at(a.ids, row * a.ldi + k);
                    const int64_t at = row * a.ldt + k;
                    av[u] = a.teacher_bf16 ? __uint_as_float(static_cast<const uint16_t*>(a.teacher)[at])
                                           : static_cast<const float*>(a.teacher)[at];
                }
            }
        }
        const T* z = static_cast<const T*>(a.z) + row * a.ldz;
        const Span sp = span_of(z, V, rank, C);
        // the unaligned ends, an element a thread: the head with the first CTA, the tail with the last
        if (rank == 0 && tid < sp.head) edge = z[tid];
        if (rank == C - 1 && tid >= 8 && tid < 8 + sp.tail) edge = z[sp.head + sp.elems + tid - 8];
    };
    if (first < a.rows) ahead(first);
    for (int64_t row = first; row < a.rows; row += step) {
        const T* z = static_cast<const T*>(a.z) + row * a.ldz;
        T* dz = grad ? static_cast<T*>(a.dz) + row * a.lddz : nullptr;
        const Span sp = span_of(z, V, rank, C);
        const int nv = sp.v1 - sp.v0;
        const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
        uint4* slot = reinterpret_cast<uint4*>(slots + static_cast<size_t>(s) * a.slot_bytes);
        const Side now = side;
        bool counts = is_live<K>(a, now);
        const int32_t tok = K != kDistill || a.labels.p ? token_of<K>(a, now) : -1;
        int32_t eid[kEntries];
        float ea[kEntries], ez[kEntries];
        const bool has_edge = (rank == 0 && tid < sp.head) || (rank == C - 1 && tid >= 8 && tid < 8 + sp.tail);
        const float e0 = counts && has_edge ? load(&edge) : -CUDART_INF_F;
        // logits at the listed ids: read here, before any CTA of the cluster overwrites them (dz may be z)
        float zt = 0.f;
        if (counts && tok >= 0) zt = load(z + tok);
        if (K == kDistill) {
#pragma unroll
            for (int u = 0; u < kEntries; ++u) {
                eid[u] = counts && tid + u * nt < a.topk ? index_of(id[u], a.ids.wide, V) : -1;
                ea[u] = eid[u] < 0 ? -CUDART_INF_F : a.teacher_bf16 ? __uint_as_float(__float_as_uint(av[u]) << 16) : av[u];
                ez[u] = eid[u] >= 0 ? load(z + eid[u]) : 0.f;
            }
        }
        if (row + step < a.rows) ahead(row + step);

        wait(smem_u32(&full_bar[s]), use, abort, a.err);
        // ---- statistics
        Stat st{e0, 0.f, 0.f};
        uint64_t kept[kKeep][P];
        float ref = 0.f;                          // what this thread's exponentials are relative to
        if (counts && HELD) {
            uint4 u[kHeld];
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                const int v = tid + q * nt;
                u[q] = v < nv ? slot[v] : Vec<T>::none();
                st.m = fmaxf(st.m, Vec<T>::top(u[q]));
            }
            ref = st.m == -CUDART_INF_F ? 0.f : st.m;
            const uint64_t nr = pack2(-ref, -ref);
            uint64_t s2[2] = {0, 0}, t2[2] = {0, 0};
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                uint64_t x[P];
                Vec<T>::get(u[q], x);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const uint64_t d = add2(x[i], nr), e = exp2_2(mul2(d, c2));
                    s2[i & 1] = add2(s2[i & 1], e);
                    if (two) t2[i & 1] = add2(t2[i & 1], exp2_2(mul2(d, l2)));
                    if (kKeep > 1) kept[q][i] = e;
                }
            }
            float x, y;
            unpack2(add2(s2[0], s2[1]), x, y);
            st.s = x + y + exp2_fast((e0 - ref) * c);
            if (two) {
                unpack2(add2(t2[0], t2[1]), x, y);
                st.s1 = x + y + exp2_fast((e0 - ref) * kLog2e);
            }
        } else if (counts) {
            uint64_t s2 = 0, t2 = 0;
            for (int v = tid; v < nv; v += nt) st.m = fmaxf(st.m, Vec<T>::top(slot[v]));
            ref = st.m == -CUDART_INF_F ? 0.f : st.m;
            const uint64_t nr = pack2(-ref, -ref);
            for (int v = tid; v < nv; v += nt) {
                uint64_t x[P];
                Vec<T>::get(slot[v], x);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const uint64_t d = add2(x[i], nr);
                    s2 = add2(s2, exp2_2(mul2(d, c2)));
                    if (two) t2 = add2(t2, exp2_2(mul2(d, l2)));
                }
            }
            float x, y;
            unpack2(s2, x, y);
            st.s = x + y + exp2_fast((e0 - ref) * c);
            if (two) {
                unpack2(t2, x, y);
                st.s1 = x + y + exp2_fast((e0 - ref) * kLog2e);
            }
        }
        const float m_own = st.m;
        st = warp_merge(st, c, two);
        Top tp{-CUDART_INF_F, 0.f, 0.f};
        if (K == kDistill && warp * 32 < a.topk) {
#pragma unroll
            for (int u = 0; u < kEntries; ++u) tp.m = fmaxf(tp.m, ea[u]);
#pragma unroll
            for (int u = 0; u < kEntries; ++u)     // an entry that the teacher rules out leaves the sums as they are
                if (ea[u] != -CUDART_INF_F) {
                    const float e = shrink(ea[u], tp.m, c);
                    tp.s += e;
                    tp.a += e * (ea[u] - tp.m);
                }
            tp = warp_merge(tp, c);
        }
        if (nw > 1) {
            if (lane == 0) {
                stat_s[par][warp] = st;
                if (K == kDistill) top_s[par][warp] = tp;
            }
            __syncthreads();
        }
        if (nw > 1) {
            st = warp_merge(lane < nw ? stat_s[par][lane] : Stat{-CUDART_INF_F, 0.f, 0.f}, c, two);
            if (K == kDistill && a.topk > 32) tp = warp_merge(lane < nw ? top_s[par][lane] : Top{-CUDART_INF_F, 0.f, 0.f}, c);
            else if (K == kDistill) tp = top_s[par][0];
        }
        if (C > 1) {
            if (warp == 0 && lane < C) {
                const uint32_t to = peer_addr(smem_u32(&cluster_s[par][rank]), lane);
                asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\tst.shared::cluster.f32 [%0+8], %3;"
                             ::"r"(to), "f"(st.m), "f"(st.s), "f"(st.s1) : "memory");
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(smem_u32(&x_bar[par]), lane)) : "memory");
            }
            wait(smem_u32(&x_bar[par]), xuse, abort, a.err);
            st = warp_merge(lane < C ? cluster_s[par][lane] : Stat{-CUDART_INF_F, 0.f, 0.f}, c, two);
        }
        if (st.s == 0.f) counts = false;
        if (!two) st.s1 = st.s;

        // ---- the row's loss and the factors of its gradient: dense exp2((z - m) c) + dense1 exp2((z - m) log2 e),
        // less what is listed at single ids
        const float ln_s = logf(st.s);
        float dense = 0.f, dense1 = 0.f, at_tok = 0.f;
        int n = 0, top = 0;                        // listed entries; the label is the last, past `top` teacher's
        if (K == kDistill) {
            const bool soft = counts && tp.s != 0.f, hard = counts && tok >= 0 && a.hard != 0.f;
            const float f = now.w * a.soft * a.inv_tau;
            if (soft) { dense = f / st.s; n = top = a.topk; }
            const float inv = 1.f / tp.s;
            float zq = 0.f;
#pragma unroll
            for (int u = 0; u < kEntries; ++u) {
                const int k = tid + u * nt;
                if (k < n) {
                    const float e = ea[u] == -CUDART_INF_F ? 0.f : exp2_fast((ea[u] - tp.m) * c) * inv;
                    id_s[k] = eid[u];
                    q_s[k] = f * e;
                    if (e != 0.f) zq += e * (ez[u] - st.m);
                }
            }
            if (warp * 32 < a.topk) {
#pragma unroll
                for (int d = 16; d; d >>= 1) zq += __shfl_xor_sync(~0u, zq, d);
            }
            if (lane == 0) zq_s[warp] = zq;
            if (hard) {
                at_tok = now.w * a.hard;
                dense1 = at_tok / st.s1;
                if (tid == 0) { id_s[n] = tok; q_s[n] = at_tok; }
                ++n;
                if (!two) { dense += dense1; dense1 = 0.f; }
            }
            __syncthreads();
            if (tid == 0 && rank == 0) {
                float loss = 0.f;
                if (soft) {
                    float z_sum = 0.f;
                    for (int w = 0; w < nw && w * 32 < a.topk; ++w) z_sum += zq_s[w];
                    loss = a.soft * ((tp.a * inv * a.inv_tau - logf(tp.s)) - (z_sum * a.inv_tau - ln_s));
                }
                if (hard) loss += a.hard * (logf(st.s1) - (zt - st.m));
                a.row_loss[row] = loss;
            }
        } else {
            const float lp = counts ? (zt - st.m) * a.inv_tau - ln_s : 0.f;
            if (K == kPolicy) {
                float loss = 0.f, slope = 0.f;
                if (counts) {
                    const float A = now.adv, ratio = expf(lp - now.old);
                    loss = -fminf(ratio * A, fminf(fmaxf(ratio, a.clip_lo), a.clip_hi) * A);
                    if (isnan(ratio * A)) loss = ratio * A;
                    slope = (A > 0.f ? ratio > a.clip_hi : ratio < a.clip_lo) ? 0.f : -A * ratio;
                    if (a.ref_logp) {
                        const float e = expm1f(now.ref - lp);
                        loss += a.kl * (e - (now.ref - lp));
                        slope -= a.kl * e;
                    }
                }
                at_tok = -slope * now.w * a.inv_tau;
                dense = counts ? at_tok / st.s : 0.f;
                if (tid == 0 && rank == 0) { a.row_loss[row] = loss; a.logp[row] = lp; }
            } else if (tid == 0 && rank == 0) {
                a.logp[row] = lp;
                a.lse[row] = counts ? st.m + ln_s : CUDART_INF_F;
                a.coef[row] = 0.f;
            }
        }

        // ---- the gradient, over the logits
        if (grad) {
            auto at = [&](float x) {
                const float d = x - st.m;
                float g = dense * exp2_fast(d * c);
                if (two) g += dense1 * exp2_fast(d * kLog2e);
                return g;
            };
            const uint64_t nm = pack2(-st.m, -st.m), dd = pack2(dense, dense), dd1 = pack2(dense1, dense1);
            if (counts && HELD) {
                const float f = dense * shrink(m_own, st.m, c);
                const uint64_t ff = pack2(f, f);
#pragma unroll
                for (int q = 0; q < kKeep; ++q) {
                    const int v = tid + q * nt;
                    if (v < nv) {
                        uint64_t x[P];
                        if (two) Vec<T>::get(slot[v], x);
#pragma unroll
                        for (int i = 0; i < P; ++i) {
                            const uint64_t g = mul2(ff, kept[q][i]);
                            x[i] = two ? fma2(dd1, exp2_2(mul2(add2(x[i], nm), l2)), g) : g;
                        }
                        slot[v] = Vec<T>::put(x);
                    }
                }
            } else if (counts) {
                for (int v = tid; v < nv; v += nt) {
                    uint64_t x[P];
                    Vec<T>::get(slot[v], x);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const uint64_t d = add2(x[i], nm);
                        x[i] = mul2(dd, exp2_2(mul2(d, c2)));
                        if (two) x[i] = fma2(dd1, exp2_2(mul2(d, l2)), x[i]);
                    }
                    slot[v] = Vec<T>::put(x);
                }
            } else {
                for (int v = tid; v < nv; v += nt) slot[v] = make_uint4(0, 0, 0, 0);
            }
            if (rank == 0 && tid < sp.head) store(dz + tid, counts ? at(e0) : 0.f);
            if (rank == C - 1 && tid >= 8 && tid < 8 + sp.tail) store(dz + sp.head + sp.elems + tid - 8, counts ? at(e0) : 0.f);
            // where an id lies: in this CTA's part of the slot, at an end that this CTA writes, or elsewhere
            T* mine = reinterpret_cast<T*>(slot);
            auto place = [&](int32_t v, int& in_slot, int& at_edge) {
                const int b = v - sp.head - sp.v0 * E;
                in_slot = v >= sp.head && b >= 0 && b < nv * E ? b : -1;
                at_edge = rank == 0 && v < sp.head ? v : rank == C - 1 && v >= sp.head + sp.elems ? 8 + v - sp.head - sp.elems : -1;
            };
            if (K == kPolicy && counts) {
                int b, e;
                place(tok, b, e);
                if (b >= 0 && tid == (b / E) % nt) store(mine + b, at(zt) - at_tok);
                if (e >= 0 && tid == e) store(dz + tok, at(zt) - at_tok);
            }
            if (K == kDistill && n > 0) {
                // each listed entry marks its place; where all find their own mark no id is listed twice
                __syncthreads();
                int b[kEntries + 1], e[kEntries + 1], who[kEntries + 1];
                float zz[kEntries + 1];
#pragma unroll
                for (int u = 0; u <= kEntries; ++u) {
                    const bool is_tok = u == kEntries;
                    const int k = is_tok ? (tid == 0 ? top : n) : tid + u * nt;
                    who[u] = -1;
                    b[u] = e[u] = -1;
                    zz[u] = is_tok ? zt : ez[u < kEntries ? u : 0];
                    if (is_tok ? k < n : k < top) {
                        const int32_t v = id_s[k];
                        if (v >= 0) {
                            place(v, b[u], e[u]);
                            if (b[u] >= 0 || e[u] >= 0) who[u] = k;
                            if (b[u] >= 0) *reinterpret_cast<uint16_t*>(mine + b[u]) = static_cast<uint16_t>(k);
                            if (e[u] >= 0) edge_s[e[u]] = k;
                        }
                    }
                }
                __syncthreads();
                bool twice = false;
#pragma unroll
                for (int u = 0; u <= kEntries; ++u) {
                    if (b[u] >= 0) twice |= *reinterpret_cast<const uint16_t*>(mine + b[u]) != who[u];
                    if (e[u] >= 0) twice |= edge_s[e[u]] != who[u];
                }
                twice = __syncthreads_or(twice);
#pragma unroll
                for (int u = 0; u <= kEntries; ++u) {
                    if (who[u] < 0) continue;
                    float g = q_s[who[u]];
                    if (twice) {
                        g = 0.f;
                        const int32_t v = id_s[who[u]];
                        for (int j = 0; j < n; ++j) g += id_s[j] == v ? q_s[j] : 0.f;
                    }
                    if (b[u] >= 0) store(mine + b[u], at(zz[u]) - g);
                    else store(dz + id_s[who[u]], at(zz[u]) - g);
                }
            }
            if (!same) {
                // the gradient's rows lie otherwise on 16 bytes than the logits': element by element
                __syncthreads();
                T* to = dz + sp.head + static_cast<int64_t>(sp.v0) * E;
                for (int q = tid; q < nv * E; q += nt) to[q] = mine[q];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncthreads();
        if (tid == 0) {
            if (grad) {
                if (nv > 0 && same)
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                                 ::"l"(dz + sp.head + static_cast<int64_t>(sp.v0) * E), "r"(smem_u32(slot)), "r"(static_cast<uint32_t>(nv) * 16u) : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                if (S > 1) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            fill();
        }
        if (++s == S) { s = 0; use ^= 1u; }
        if (par) xuse ^= 1u;
        par ^= 1;
    }
    if (tid == 0) {
        if (grad) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        if (*abort)                                   // let the copies already issued land
            for (int q = 0; q < S; ++q)
                if (filled >> q & 1u)
                    for (int it = 0; it < 4000000 && !try_wait(smem_u32(&full_bar[q]), fill_par >> q & 1u); ++it) __nanosleep(64);
    }
    // no CTA of a cluster leaves while another may still write to its shared memory
    if (C > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

constexpr int kThreads = 512;

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

// Shape of a launch: how many CTAs share a row, their slots and threads.
template <int K>
cudaError_t rows_launch(RowArgs a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, row_bytes = a.vocab * es;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const int64_t vecs = (row_bytes + 15) / 16;
    int C = 1;
    while (C < kMaxCluster && (vecs + C - 1) / C * 16 > kSlotMax) C *= 2;
    // few rows: more CTAs a row, as long as each has 4 KiB of it
    while (C < kMaxCluster && a.rows * C * 2 <= sms && row_bytes / (2 * C) >= 4096) C *= 2;
    a.cluster = C;
    a.slot_bytes = static_cast<uint32_t>((vecs + C - 1) / C * 16);
    a.slots = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(3, kRingMax / a.slot_bytes)));
    const size_t smem = static_cast<size_t>(a.slots) * a.slot_bytes;
    const bool held = a.slot_bytes <= kSlotMax;
    int warps = held ? static_cast<int>((a.slot_bytes / 16 + 32 * kHeld - 1) / (32 * kHeld)) : kMaxWarps;
    if (K == kDistill) warps = std::max(warps, (a.topk + 32 * kEntries - 1) / (32 * kEntries));
    const int per_sm = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({16, kRingMax / static_cast<int64_t>(smem + 1024), 16 / warps})));
    const int64_t groups = std::min<int64_t>(a.rows, std::max<int64_t>(1, static_cast<int64_t>(sms) * per_sm / C));
    auto kernel = dtype == GLR_BF16 ? (held ? rows_kernel<K, __nv_bfloat16, true> : rows_kernel<K, __nv_bfloat16, false>)
                                    : (held ? rows_kernel<K, float, true> : rows_kernel<K, float, false>);
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kRingMax))) != cudaSuccess) return e;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = C; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = static_cast<unsigned>(groups * C); cfg.blockDim = warps * 32; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
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
