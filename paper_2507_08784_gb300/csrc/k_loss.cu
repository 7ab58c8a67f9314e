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
// Natural logarithm by the hardware's of base 2: within 2^-22 absolute near 1, 2^-22 relative elsewhere.
__device__ __forceinline__ float log_fast(float x) {
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y * 0.6931471805599453f;
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
template <bool TWO>
__device__ __forceinline__ Stat warp_merge(Stat x, float c) {
    Stat r;
    r.m = warp_max(x.m);
    r.s = warp_sum(x.s * shrink(x.m, r.m, c));
    r.s1 = TWO ? warp_sum(x.s1 * shrink(x.m, r.m, kLog2e)) : 0.f;
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

// `peers`: what other CTAs of the cluster wrote before they arrived is to be seen.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity, bool peers) {
    uint32_t done;
    if (peers)
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    else
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Bounded wait.  One that gives up raises the CTA's abort flag and counts; from then on every wait of the
// CTA returns at once, so that its threads still meet at their barriers and leave together.
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, bool peers, volatile int* abort, int* err) {
    for (int it = 0; it < 16000000; ++it) {
        if (try_wait(bar, parity, peers)) return;
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
struct __align__(16) Span {
    int head, elems;                         // elements before the vectors, and in them
    int v0, nv;                              // vectors [v0, v0 + nv) are this CTA's
};
template <class T>
__device__ __forceinline__ Span span_of(const T* z, int vocab, int rank, int shift) {
    constexpr int E = Vec<T>::kElems;
    Span s;
    s.head = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(T));
    s.head = s.head < vocab ? s.head : vocab;
    const int n = (vocab - s.head) / E, per = (n + (1 << shift) - 1) >> shift;
    s.elems = n * E;
    s.v0 = min(rank * per, n);
    s.nv = min(s.v0 + per, n) - s.v0;
    return s;
}
// What one thread prepares for all of them, a row ahead.
struct __align__(16) Row {
    Span span;
    float w, adv, old, ref;
    float zt;                                // the logit at the row's token or label
    int32_t tok;                             // -1: none
    int live, pad;
};

constexpr int64_t kSlotMax = kMaxWarps * 32 * kHeld * 16;    // of a row a CTA: 64 KiB, three slots fit
constexpr int64_t kRingMax = 208 * 1024;

// HELD: a slot has at most kHeld vectors a thread, and the exponentials of the statistics stay in registers
// for the gradient; else (rows of more than eight such slots) they are formed again.  TWO: a hard term beside
// tau != 1, so that the sums are kept at two temperatures.
//
// A row is a chain of short steps between three barriers, and what every warp does for itself in it is paid
// sixteen times over: so one thread prepares the row data for all, another one copies, only the warps that
// hold teacher entries look at them, and whatever comes from memory is asked for a row before it is used.
template <int K, class T, bool HELD, bool TWO>
__global__ void __launch_bounds__(kMaxWarps * 32) rows_kernel(const __grid_constant__ RowArgs a) {
    chain_begin();
    constexpr int E = Vec<T>::kElems, P = E / 2;
    constexpr int kKeep = HELD && K != kLogProb ? kHeld : 1;
    constexpr bool D = K == kDistill;
    extern __shared__ __align__(128) uint8_t slots[];
    __shared__ __align__(8) uint64_t full_bar[kMaxSlots], x_bar[2];
    // by the row's parity: a warp may be a row ahead of one that still reads
    __shared__ Row row_s[2];
    __shared__ Stat stat_s[2][kMaxWarps], cluster_s[2][kMaxCluster];
    __shared__ Top top_s[2][D ? kMaxWarps : 1];
    __shared__ float zq_s[D ? kMaxWarps : 1];
    __shared__ int32_t id_s[D ? GLR_MAX_TOPK + 1 : 1];
    __shared__ float q_s[D ? GLR_MAX_TOPK + 1 : 1];
    __shared__ int abort_flag;
    const int nt = blockDim.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nw = nt >> 5;
    const int C = 1 << a.cluster_shift, S = a.slots, V = static_cast<int>(a.vocab);
    uint32_t rank = 0;
    if (C > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int64_t first = blockIdx.x >> a.cluster_shift, step = gridDim.x >> a.cluster_shift;
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
    const float c = a.inv_tau * kLog2e;
    const uint64_t c2 = pack2(c, c), l2 = pack2(kLog2e, kLog2e);
    auto logits = [&](int64_t row) { return static_cast<const T*>(a.z) + row * a.ldz; };

    // The copying thread fills the slots, and writes them back once every thread is done with a row.
    const bool copier = tid == (nw >> 1) * 32;
    int64_t next = first;
    Side ask{};                                       // the next row to fill: whether it is read
    int fs = 0;
    uint32_t filled = 0, fill_par = 0;                // per slot (bit q): filled at all, parity of the last fill
    auto fill = [&]() {
        if (next >= a.rows) return;
        const T* z = logits(next);
        const Span sp = span_of(z, V, rank, a.cluster_shift);
        const uint32_t bytes = is_live<K>(a, ask) ? static_cast<uint32_t>(sp.nv) * 16u : 0u;
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
    // with a gradient the slot of the row before is filled in the middle of this one (S = 1: its own, at the end)
    if (copier) {
        if (first < a.rows) ask = side_at<K>(a, first, false);
        for (int q = 0; q < (grad && S > 1 ? S - 1 : S); ++q) fill();
    }
    // The preparing thread: `side` holds the row after the one in progress, the logit at its token is on the way.
    const bool preparer = tid == (nw - 1) * 32;
    Side side{};
    T zt_raw{};
    auto look_up = [&](int64_t row) {                 // side is that row's: its token's logit
        const int32_t tok = K != kDistill || a.labels.p ? token_of<K>(a, side) : -1;
        if (tok >= 0 && is_live<K>(a, side)) zt_raw = logits(row)[tok];
    };
    auto prepare = [&](int64_t row, Row& r) {
        r.span = span_of(logits(row), V, rank, a.cluster_shift);
        r.w = side.w; r.adv = side.adv; r.old = side.old; r.ref = side.ref;
        r.tok = K != kDistill || a.labels.p ? token_of<K>(a, side) : -1;
        r.live = is_live<K>(a, side);
        r.zt = load(&zt_raw);
    };
    Side after{};                                     // and the row after that
    if (preparer && first < a.rows) {
        side = side_at<K>(a, first, true);
        look_up(first);
        prepare(first, row_s[0]);
        if (first + step < a.rows) side = side_at<K>(a, first + step, true);
    }
    // Teacher entries, 32 kEntries a warp: entry k = warp 32 kEntries + 32 u + lane.
    const int k0 = warp * 32 * kEntries + lane;
    const bool entries = D && warp * 32 * kEntries < a.topk;
    Word id[kEntries];
    float av[kEntries];                               // bf16 teacher logits as their bits
    auto ask_entries = [&](int64_t row) {
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            const int k = k0 + 32 * u;
            if (k < a.topk) {
                id[u] = word_at(a.ids, row * a.ldi + k);
                const int64_t at = row * a.ldt + k;
                av[u] = a.teacher_bf16 ? __uint_as_float(static_cast<const uint16_t*>(a.teacher)[at]) : static_cast<const float*>(a.teacher)[at];
            }
        }
    };
    if (entries && first < a.rows) ask_entries(first);
    __syncthreads();

    int s = 0, par = 0;
    uint32_t use = 0, xuse = 0;
    for (int64_t row = first; row < a.rows; row += step) {
        const Row now = row_s[par];
        const Span sp = now.span;
        const int nv = sp.nv;
        bool counts = now.live;
        uint4* slot = reinterpret_cast<uint4*>(slots + static_cast<size_t>(s) * a.slot_bytes);
        const bool more = row + step < a.rows;
        // ---- ask for what comes from memory.  Logits of this row are read here, before any CTA of the cluster
        // overwrites them (dz may be z)
        int32_t eid[kEntries];
        float ea[kEntries];
        T ez_raw[kEntries];                           // widened where they are used
        if (entries) {
            const T* z = logits(row);
#pragma unroll
            for (int u = 0; u < kEntries; ++u) {
                const int k = k0 + 32 * u;
                eid[u] = counts && k < a.topk ? index_of(id[u], a.ids.wide, V) : -1;
                ea[u] = eid[u] < 0 ? -CUDART_INF_F : a.teacher_bf16 ? __uint_as_float(__float_as_uint(av[u]) << 16) : av[u];
                if (eid[u] >= 0) ez_raw[u] = z[eid[u]];
                if (k < a.topk) id_s[k] = eid[u];
            }
            if (more) ask_entries(row + step);
        }
        const bool hard = D && counts && now.tok >= 0 && a.hard != 0.f;
        if (D && tid == 0) id_s[a.topk] = hard ? now.tok : -1;
        // the unaligned ends, an element a thread: the head with the first CTA, the tail with the last
        T edge{};
        int at_end = -1;                              // this thread's element of the ends
        if (warp == 0) {
            if (rank == 0 && lane < sp.head) at_end = lane;
            if (rank == C - 1 && lane >= 8 && lane < 8 + V - sp.head - sp.elems) at_end = sp.head + sp.elems + lane - 8;
            if (counts && at_end >= 0) edge = logits(row)[at_end];
        }
        if (preparer && more) {
            look_up(row + step);
            if (row + 2 * step < a.rows) after = side_at<K>(a, row + 2 * step, true);
        }

        wait(smem_u32(&full_bar[s]), use, false, abort, a.err);
        // ---- statistics
        Stat st{-CUDART_INF_F, 0.f, 0.f};
        uint64_t kept[kKeep][P];
        if (counts && HELD) {
            uint4 u[kHeld];
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                const int v = tid + q * nt;
                u[q] = v < nv ? slot[v] : Vec<T>::none();
                st.m = fmaxf(st.m, Vec<T>::top(u[q]));
            }
            const float ref = st.m == -CUDART_INF_F ? 0.f : st.m;
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
                    if (TWO) t2[i & 1] = add2(t2[i & 1], exp2_2(mul2(d, l2)));
                    if (kKeep > 1) kept[q][i] = e;
                }
            }
            float x, y;
            unpack2(add2(s2[0], s2[1]), x, y);
            st.s = x + y;
            unpack2(add2(t2[0], t2[1]), x, y);
            st.s1 = x + y;
        } else if (counts) {
            uint64_t s2 = 0, t2 = 0;
            for (int v = tid; v < nv; v += nt) st.m = fmaxf(st.m, Vec<T>::top(slot[v]));
            const float ref = st.m == -CUDART_INF_F ? 0.f : st.m;
            const uint64_t nr = pack2(-ref, -ref);
            for (int v = tid; v < nv; v += nt) {
                uint64_t x[P];
                Vec<T>::get(slot[v], x);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const uint64_t d = add2(x[i], nr);
                    s2 = add2(s2, exp2_2(mul2(d, c2)));
                    if (TWO) t2 = add2(t2, exp2_2(mul2(d, l2)));
                }
            }
            float x, y;
            unpack2(s2, x, y);
            st.s = x + y;
            unpack2(t2, x, y);
            st.s1 = x + y;
        }
        const float m_own = st.m;                     // what this thread's exponentials are relative to
        const float e0 = load(&edge);
        if (warp == 0 && counts && at_end >= 0) {     // one more element
            const float m = fmaxf(st.m, e0), r = m == -CUDART_INF_F ? 0.f : m;
            st.s = st.s * shrink(st.m, m, c) + exp2_fast((e0 - r) * c);
            if (TWO) st.s1 = st.s1 * shrink(st.m, m, kLog2e) + exp2_fast((e0 - r) * kLog2e);
            st.m = m;
        }
        st = warp_merge<TWO>(st, c);
        Top tp{-CUDART_INF_F, 0.f, 0.f};
        if (entries) {
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
        if (lane == 0) {
            stat_s[par][warp] = st;
            if (entries) top_s[par][warp] = tp;
        }
        __syncthreads();
        if (copier && grad && S > 1) {                 // the slot of the row before has been written back by now
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            fill();
        }
        if (nw > 1) st = warp_merge<TWO>(lane < nw ? stat_s[par][lane] : Stat{-CUDART_INF_F, 0.f, 0.f}, c);
        if (C > 1 && warp == 0 && lane < C) {
            const uint32_t to = peer_addr(smem_u32(&cluster_s[par][rank]), lane);
            asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\tst.shared::cluster.f32 [%0+8], %3;"
                         ::"r"(to), "f"(st.m), "f"(st.s), "f"(st.s1) : "memory");
            asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(smem_u32(&x_bar[par]), lane)) : "memory");
        }
        // ---- while the peers' sums come in: the teacher's sums, and whether an id is listed twice
        const int top = a.topk, n = D && counts ? top + 1 : 0;
        bool twice = false;
        if (D && counts) {
            if (top > 32 * kEntries) tp = warp_merge(lane * 32 * kEntries < top ? top_s[par][lane & (kMaxWarps - 1)] : Top{-CUDART_INF_F, 0.f, 0.f}, c);
            else if (top > 0) tp = top_s[par][0];
            if (grad) {
                // entry k against the earlier ones: 2^dup_shift threads an entry
                const int parts = 1 << a.dup_shift;
                for (int k = tid >> a.dup_shift; k < n; k += nt >> a.dup_shift) {
                    const int32_t v = id_s[k];
                    for (int j = tid & (parts - 1); j < k; j += parts) twice |= id_s[j] == v && v >= 0;
                }
            }
        }
        if (C > 1) {
            wait(smem_u32(&x_bar[par]), xuse, true, abort, a.err);
            st = warp_merge<TWO>(lane < C ? cluster_s[par][lane] : Stat{-CUDART_INF_F, 0.f, 0.f}, c);
        }
        if (st.s == 0.f) counts = false;
        if (!TWO) st.s1 = st.s;

        // ---- the row's loss and the factors of its gradient: dense exp2((z - m) c) + dense1 exp2((z - m) log2 e),
        // less what is listed at single ids
        const float inv_s = __fdividef(1.f, st.s), zt = now.zt;
        float dense = 0.f, dense1 = 0.f, at_tok = 0.f, q[kEntries] = {};
        if (K == kDistill) {
            const bool soft = counts && tp.s != 0.f;
            const float f = now.w * a.soft * a.inv_tau, inv = 1.f / tp.s;
            if (soft) dense = f * inv_s;
            if (hard && counts) {
                at_tok = now.w * a.hard;
                dense1 = at_tok / st.s1;
                if (!TWO) { dense += dense1; dense1 = 0.f; }
            }
            if (entries) {
                float zq = 0.f;
#pragma unroll
                for (int u = 0; u < kEntries; ++u) {
                    const float e = !soft || ea[u] == -CUDART_INF_F ? 0.f : exp2_fast((ea[u] - tp.m) * c) * inv;
                    q[u] = f * e;
                    if (k0 + 32 * u < top) q_s[k0 + 32 * u] = q[u];
                    if (e != 0.f) zq += e * (load(&ez_raw[u]) - st.m);
                }
                zq = warp_sum(zq);
                if (lane == 0) zq_s[warp] = zq;
            }
            if (tid == 0) q_s[top] = at_tok;
        } else {
            const float lp = counts ? (zt - st.m) * a.inv_tau - log_fast(st.s) : 0.f;
            if (K == kPolicy) {
                float loss = 0.f, slope = 0.f;
                if (counts) {
                    const float A = now.adv, ratio = exp2_fast((lp - now.old) * kLog2e);
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
                dense = counts ? at_tok * inv_s : 0.f;
                if (tid == 0 && rank == 0) { a.row_loss[row] = loss; a.logp[row] = lp; }
            } else if (tid == 0 && rank == 0) {
                a.logp[row] = lp;
                a.lse[row] = counts ? st.m + log_fast(st.s) : CUDART_INF_F;
                a.coef[row] = 0.f;
            }
        }

        // ---- the gradient, over the logits
        T* mine = reinterpret_cast<T*>(slot);
        auto at = [&](float x) {
            const float d = x - st.m;
            float g = dense * exp2_fast(d * c);
            if (TWO) g += dense1 * exp2_fast(d * kLog2e);
            return g;
        };
        // the place of an id in this CTA's part of the row, or negative
        auto place = [&](int32_t v) {
            const int b = v - sp.head - sp.v0 * E;
            return b < nv * E ? b : -1;
        };
        auto row_of = [&]() { return static_cast<T*>(a.dz) + row * a.lddz; };
        auto is_end = [&](int32_t v) { return (rank == 0 && v < sp.head) || (rank == C - 1 && v >= sp.head + sp.elems); };
        if (grad) {
            if (counts && HELD) {
                const float f = dense * shrink(m_own, st.m, c);
                const uint64_t ff = pack2(f, f), nm = pack2(-st.m, -st.m), dd1 = pack2(dense1, dense1);
#pragma unroll
                for (int j = 0; j < kKeep; ++j) {
                    const int v = tid + j * nt;
                    if (v < nv) {
                        uint64_t x[P];
                        if (TWO) Vec<T>::get(slot[v], x);
#pragma unroll
                        for (int i = 0; i < P; ++i) {
                            const uint64_t g = mul2(ff, kept[j][i]);
                            x[i] = TWO ? fma2(dd1, exp2_2(mul2(add2(x[i], nm), l2)), g) : g;
                        }
                        slot[v] = Vec<T>::put(x);
                    }
                }
            } else if (counts) {
                const uint64_t nm = pack2(-st.m, -st.m), dd = pack2(dense, dense), dd1 = pack2(dense1, dense1);
                for (int v = tid; v < nv; v += nt) {
                    uint64_t x[P];
                    Vec<T>::get(slot[v], x);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const uint64_t d = add2(x[i], nm);
                        x[i] = mul2(dd, exp2_2(mul2(d, c2)));
                        if (TWO) x[i] = fma2(dd1, exp2_2(mul2(d, l2)), x[i]);
                    }
                    slot[v] = Vec<T>::put(x);
                }
            } else {
                for (int v = tid; v < nv; v += nt) slot[v] = make_uint4(0, 0, 0, 0);
            }
            if (at_end >= 0) {
                float g = counts ? at(e0) : 0.f;
                if (K == kPolicy && counts && at_end == now.tok) g -= at_tok;
                store(row_of() + at_end, g);
            }
            if (K == kPolicy && counts) {              // by the thread that wrote the token's vector
                const int b = place(now.tok);
                int v = b / E;
                if (HELD) {
#pragma unroll
                    for (int j = 1; j < kHeld; ++j) v -= v >= nt ? nt : 0;
                } else {
                    v %= nt;
                }
                if (b >= 0 && v == tid) store(mine + b, at(zt) - at_tok);
            }
        }
        if (K == kDistill) {
            // every thread's part of the gradient is written before single entries are: the slot's, and the ends'
            twice = __syncthreads_or(twice);
            if (tid == 0 && rank == 0) {
                float loss = 0.f;
                if (counts && tp.s != 0.f) {
                    float z_sum = 0.f;
                    for (int w = 0; w * 32 * kEntries < top; ++w) z_sum += zq_s[w];
                    loss = a.soft * ((tp.a / tp.s * a.inv_tau - log_fast(tp.s)) - (z_sum * a.inv_tau - log_fast(st.s)));
                }
                if (hard && counts) loss += a.hard * (log_fast(st.s1) - (zt - st.m));
                a.row_loss[row] = loss;
            }
            if (grad && counts && (entries || tid == 0)) {
                auto single = [&](int32_t v, float g, float z) {
                    if (v < 0) return;
                    const int b = place(v);
                    if (b < 0 && !is_end(v)) return;
                    if (twice) {
                        g = 0.f;
                        for (int j = 0; j < n; ++j) g += id_s[j] == v ? q_s[j] : 0.f;
                    }
                    store(b >= 0 ? mine + b : row_of() + v, at(z) - g);
                };
                if (entries) {
#pragma unroll
                    for (int u = 0; u < kEntries; ++u) single(eid[u], q[u], load(&ez_raw[u]));
                }
                if (tid == 0 && hard) single(now.tok, at_tok, zt);
            }
        }
        const bool same = grad && ((reinterpret_cast<uintptr_t>(logits(row)) ^ reinterpret_cast<uintptr_t>(row_of())) & 15) == 0;
        if (grad && !same) {
            // the gradient's rows lie otherwise on 16 bytes than the logits': element by element
            __syncthreads();
            T* to = row_of() + sp.head + static_cast<int64_t>(sp.v0) * E;
            for (int j = tid; j < nv * E; j += nt) to[j] = mine[j];
        }
        if (preparer && more) {
            prepare(row + step, row_s[par ^ 1]);
            side = after;
        }
        __syncthreads();
        if (copier) {
            if (grad) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // all threads' writes, before the copy reads them
                if (nv > 0 && same)
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                                 ::"l"(row_of() + sp.head + static_cast<int64_t>(sp.v0) * E), "r"(smem_u32(slot)), "r"(static_cast<uint32_t>(nv) * 16u) : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                if (S == 1) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            if (!grad || S == 1) fill();
        }
        if (++s == S) { s = 0; use ^= 1u; }
        if (par) xuse ^= 1u;
        par ^= 1;
    }
    if (copier) {
        if (grad) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        if (*abort)                                   // let the copies already issued land
            for (int q = 0; q < S; ++q)
                if (filled >> q & 1u)
                    for (int it = 0; it < 4000000 && !try_wait(smem_u32(&full_bar[q]), fill_par >> q & 1u, false); ++it) __nanosleep(64);
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
    a.cluster_shift = C == 1 ? 0 : C == 2 ? 1 : C == 4 ? 2 : 3;
    a.slot_bytes = static_cast<uint32_t>((vecs + C - 1) / C * 16);
    a.slots = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(3, kRingMax / a.slot_bytes)));
    const size_t smem = static_cast<size_t>(a.slots) * a.slot_bytes;
    const bool held = a.slot_bytes <= kSlotMax;
    int warps = held ? static_cast<int>((a.slot_bytes / 16 + 32 * kHeld - 1) / (32 * kHeld)) : kMaxWarps;
    if (K == kDistill) {
        warps = std::max(warps, (a.topk + 32 * kEntries - 1) / (32 * kEntries));
        a.dup_shift = 0;                          // threads an entry in the search for ids listed twice
        while ((a.topk + 1) << (a.dup_shift + 1) <= warps * 32) ++a.dup_shift;
    }
    const int per_sm = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({16, kRingMax / static_cast<int64_t>(smem + 1024), 16 / warps})));
    const int64_t groups = std::min<int64_t>(a.rows, std::max<int64_t>(1, static_cast<int64_t>(sms) * per_sm / C));
    const bool two = K == kDistill && a.labels.p && a.hard != 0.f && a.inv_tau != 1.f;
    auto pick = [&](auto t) {
        using T = decltype(t);
        constexpr bool D = K == kDistill;
        return held ? (two ? rows_kernel<K, T, true, D> : rows_kernel<K, T, true, false>)
                    : (two ? rows_kernel<K, T, false, D> : rows_kernel<K, T, false, false>);
    };
    auto kernel = dtype == GLR_BF16 ? pick(__nv_bfloat16()) : pick(float());
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
