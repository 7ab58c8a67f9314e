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
// reduced by the worker warps, overwritten by its own gradient and written back by a bulk copy.  The
// CTAs of a cluster exchange (m, s) over distributed shared memory.  Two service warps do everything else,
// taking rows in turn: row data, copies, teacher entries, losses, single entries.
//
// Bound by HBM on many rows (8192 rows of 131071 bf16, policy loss: 636 us, 6.7 TB/s), by the copies' and barriers'
// latency on rows of a few KiB (65536 rows of 2048 bf16: 170 us, 3.2 TB/s), and between them by both and the workers'
// arithmetic (4096 rows of 32768 bf16: 95 to 103 us, 5.3 TB/s; without a gradient 64 us, 4.2 TB/s: a slot is handed on as if
// it were written).
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

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
// Natural logarithm of a sum s >= 1: its series in s - 1 up to s = 17 / 16 (within 2^-22 of its value), else the hardware's
// logarithm of base 2, which is off by up to 2^-22: 1 to 2 % of the loss of a token predicted with 1 - 1e-5.  (logf takes the
// workers 1 to 3 % of a row: 8192 rows of 131071 bf16 645 us instead of 638, policy loss.)
__device__ __forceinline__ float log_of(float s) {
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(s));
    const float t = s - 1.f;
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.2f, -0.25f), 0.333333333f), -0.5f), 1.f);
    return fabsf(t) < 0.0625f ? p : y * 0.6931471805599453f;
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
    using Mark = uint16_t;
    static __device__ __forceinline__ void scatter(__nv_bfloat16* p, const uint4& u) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
        for (int q = 0; q < 4; ++q) { h[2 * q] = static_cast<uint16_t>(w[q]); h[2 * q + 1] = static_cast<uint16_t>(w[q] >> 16); }
    }
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
    using Mark = uint32_t;
    static __device__ __forceinline__ void scatter(float* p, const uint4& u) {
        p[0] = __uint_as_float(u.x); p[1] = __uint_as_float(u.y); p[2] = __uint_as_float(u.z); p[3] = __uint_as_float(u.w);
    }
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
template <int TWO>
__device__ __forceinline__ Stat warp_merge(Stat x, float c) {
    Stat r{};
    r.m = warp_max(x.m);
    r.s = warp_sum(x.s * shrink(x.m, r.m, c));
    r.s1 = TWO ? warp_sum(x.s1 * shrink(x.m, r.m, kLog2e)) : 0.f;
    return r;
}
constexpr int kWorkers = 14;                // warps on a row at most; two more are service warps, one of which beside a teacher's
constexpr int kMaxSlots = 3;
constexpr int kMaxCluster = 8;
constexpr int kHeld = 10;                   // 16-byte vectors of a slot whose exponentials a thread keeps in registers

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
// What a row needs beside its logits.  It is asked for well before it is looked at: an index stays as its two
// words, and nothing is compared or converted on the way, which would wait for memory.
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
__device__ __forceinline__ Side side_at(const RowArgs& a, int64_t row) {
    Side s{};
    s.w = K == kLogProb ? 1.f : a.weight ? a.weight[row] : a.share;
    s.tok = {-1, 0};
    if (K != kDistill) s.tok = word_at(a.tokens, row);
    else if (a.labels.p) s.tok = word_at(a.labels, row);
    if (K == kPolicy) {
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
// A row's data, prepared four rows ahead.
struct __align__(16) Row {
    Span span;
    float w, adv, old, ref;
    int32_t tok;                             // the row's token or label, -1: none
    int live, same, pad;                     // same: logits and gradient lie alike on 16 bytes
};
// What the workers need of a row beside its sums: the logit at its token, and whether the teacher has entries.
struct Pub { float zt; int soft; };
// A row's loss and the factors of its gradient: dense exp2((z - m) c) + dense1 exp2((z - m) log2 e), less at_tok at
// the token (distillation: and what the teacher's entries take).
struct Coef { float dense, dense1, at_tok, loss, lp; };

template <int K, int TWO>
__device__ __forceinline__ Coef coef_of(const RowArgs& a, const Row& r, const Stat& st, const Pub& pub, bool counts) {
    Coef k{};
    if (K == kDistill) {
        if (counts && pub.soft) k.dense = r.w * a.soft * a.inv_tau * __fdividef(1.f, st.s);
        if (counts && r.tok >= 0 && a.hard != 0.f) {
            k.at_tok = r.w * a.hard;
            k.dense1 = k.at_tok * __fdividef(1.f, st.s1);
            if (!TWO) { k.dense += k.dense1; k.dense1 = 0.f; }
        }
        return k;
    }
    if (!counts) return k;
    k.lp = (pub.zt - st.m) * a.inv_tau - log_of(st.s);
    if (K == kPolicy) {
        const float A = r.adv, ratio = exp2_fast((k.lp - r.old) * kLog2e);
        const float gain = A == 0.f && ratio == CUDART_INF_F ? 0.f : ratio * A;      // (the ratio may leave the range)
        k.loss = -fminf(gain, fminf(fmaxf(ratio, a.clip_lo), a.clip_hi) * A);
        if (isnan(gain)) k.loss = gain;
        float slope = (A > 0.f ? ratio > a.clip_hi : ratio < a.clip_lo) ? 0.f : -gain;
        if (a.ref_logp && a.kl != 0.f) {              // (and so may exp(e))
            const float e = expm1f(r.ref - k.lp);
            k.loss += a.kl * (e - (r.ref - k.lp));
            slope -= a.kl * e;
        }
        k.at_tok = -slope * r.w * a.inv_tau;
        k.dense = k.at_tok * __fdividef(1.f, st.s);
    }
    return k;
}

constexpr int64_t slot_max(int workers) { return int64_t(workers) * 32 * kHeld * 16; }   // of a row a CTA: 70 KiB
constexpr int64_t kRingMax = 196 * 1024;                     // three slots of 64 KiB and some bytes
constexpr int64_t kDynMax = 222 * 1024;                      // ... and a teacher's lists
constexpr int kFewEntries = 64;
constexpr int kMaxLists = 4;
// A list: ids, q and logits of a row's entries, the label last, and whether the teacher has any and sum q log q.
__host__ __device__ constexpr int list_words(int64_t topk) { return (3 * (static_cast<int>(topk) + 1) + 2 + 3) & ~3; }
// FEW (at most 64 entries): the service warps see to the teacher's entries; else a warp of its own does.
constexpr int most_workers(bool few) { return few ? kWorkers : kWorkers - 1; }

// HELD: a slot has at most kHeld vectors a worker thread, and the exponentials of the statistics stay in
// registers for the gradient; else (rows of more than eight such slots) they are formed again.  TWO: a hard
// term beside tau != 1, so that the sums are kept at two temperatures: kBoth takes two exponentials an element, and at
// tau = 2 or 4 the second is the first's square or fourth power (4096 rows
// of 32768 bf16, 64 entries, a hard term: tau = 2 126 -> 107 us, tau = 4 126 -> 111, tau = 3 126, tau = 1 103).
//
// A worker's row is: wait for the slot, sums, one barrier, the merge of all warps' sums (and of the cluster's
// CTAs), the gradient into the slot.  What each of up to fourteen warps would do for itself is paid that many
// times over, and a load's latency in this chain is lost to all of them, so the service warps do the rest, each
// for every second row i:
//   1 asks for the ends, the token's logit and the teacher's entries of row i + 2, and for the data of rows
//     i + 3 and i + 4
//   2 the ends' sums and the token's logit of row i, before the workers' barrier
//   3 the loss of row i, once its sums are there
//   4 single entries of row i's gradient, once the workers have written theirs, its write-back, and the fill of
//     its slot with row i + S (S slots)
//   5 puts down what was asked for, with the teacher's softmax
// Their code is run once a row by one warp, so that it is bound by instruction fetch: its loops are kept rolled.
// With more than 64 entries (FEW false) the latter would not be done in time: a warp of its own sees to them, ahead by
// up to four rows, and takes a worker's place (8192 rows of 131071 bf16, 128 entries: 917 -> 734 us; 4096 rows of 32768,
// 128 entries 124 -> 108, 64 entries 96 -> 101 if it did it there too).
constexpr int kBoth = 1, kSquares = 2, kFourths = 3;
// s + e^tau, and f e + f1 e^tau
template <int TWO>
__device__ __forceinline__ uint64_t power_sum(uint64_t e, uint64_t s) {
    if (TWO == kFourths) e = mul2(e, e);
    return fma2(e, e, s);
}
template <int TWO>
__device__ __forceinline__ uint64_t two_powers(uint64_t f, uint64_t f1, uint64_t e) {
    const uint64_t q = TWO == kFourths ? mul2(mul2(e, e), e) : e;
    return mul2(fma2(f1, q, f), e);
}
template <int K, class T, bool HELD, int TWO, bool FEW>
__global__ void __launch_bounds__((kWorkers + 2) * 32) rows_kernel(const __grid_constant__ RowArgs a) {
    chain_begin();
    constexpr int E = Vec<T>::kElems, P = E / 2;
    constexpr int kKeep = HELD && K != kLogProb ? kHeld : 1;
    constexpr bool D = K == kDistill;
    constexpr bool TEACH = D && !FEW;
    constexpr int kList = D && FEW ? kFewEntries + 1 : 1;     // entries subtracted at single ids; the token is the last
    extern __shared__ __align__(128) uint8_t slots[];
    __shared__ __align__(8) uint64_t full_bar[kMaxSlots], x_bar[2], fin_bar[2], dense_bar[2], list_bar[kMaxLists], read_bar[kMaxLists];
    // by the row's parity, or (row_s) its number modulo four: who writes them again has passed a barrier that
    // all readers have reached
    __shared__ Row row_s[4];
    __shared__ Stat stat_s[2][kWorkers + 1], fin_s[2];
    __shared__ __align__(16) float4 cluster_s[2][kMaxCluster];
    __shared__ Pub pub_s[2];
    __shared__ float end_s[2][16], zt_s[2];
    __shared__ int32_t id_s[2][kList], mark_s[2][16];
    __shared__ float q_s[2][kList], z_s[2][kList];
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nw = (blockDim.x >> 5) - (TEACH ? 3 : 2), nt = nw * 32;
    const int C = 1 << a.cluster_shift, S = a.slots, V = static_cast<int>(a.vocab);
    uint32_t rank = 0;
    if (C > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int64_t first = blockIdx.x >> a.cluster_shift, step = gridDim.x >> a.cluster_shift;
    volatile int* abort = &abort_flag;
    if (tid == 0) {
        abort_flag = 0;
        for (int q = 0; q < S; ++q) mbar_init(smem_u32(&full_bar[q]), 1);
        for (int q = 0; q < 2; ++q) {
            mbar_init(smem_u32(&x_bar[q]), 1);
            mbar_init(smem_u32(&fin_bar[q]), 1);
            mbar_init(smem_u32(&dense_bar[q]), nw);
        }
        if (TEACH)
            for (int q = 0; q < kMaxLists; ++q) { mbar_init(smem_u32(&list_bar[q]), 1); mbar_init(smem_u32(&read_bar[q]), 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const bool grad = K != kLogProb && a.dz != nullptr;
    const float c = a.inv_tau * kLog2e;
    const uint64_t c2 = pack2(c, c), l2 = pack2(kLog2e, kLog2e);
    auto logits = [&](int64_t row) { return static_cast<const T*>(a.z) + row * a.ldz; };
    auto gradient = [&](int64_t row) { return static_cast<T*>(a.dz) + row * a.lddz; };
    auto prepare = [&](int64_t row, int it, const Side& side) {
        Row r{};
        r.span = span_of(logits(row), V, rank, a.cluster_shift);
        r.w = side.w; r.adv = side.adv; r.old = side.old; r.ref = side.ref;
        r.tok = !D || a.labels.p ? token_of<K>(a, side) : -1;
        r.live = is_live<K>(a, side);
        r.same = ((reinterpret_cast<uintptr_t>(logits(row)) ^ reinterpret_cast<uintptr_t>(gradient(row))) & 15) == 0;
        row_s[it & 3] = r;
    };
    if (warp == nw && lane < 4 && first + lane * step < a.rows) prepare(first + lane * step, lane, side_at<K>(a, first + lane * step));
    __syncthreads();
    if (C > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");

    // row i's list (i mod a.lists; a power of two of them)
    auto list_of = [&](int i) {
        return reinterpret_cast<int32_t*>(slots + static_cast<size_t>(S) * a.slot_bytes) + (i & (a.lists - 1)) * list_words(a.topk);
    };
    const int n1 = a.topk + 1;
    int s = 0, it = 0;
    uint32_t use = 0, xuse = 0;
    if (TEACH && warp == nw + 2) {
        // The teacher's warp, as far ahead as there are lists: a row's entries are asked for a row earlier, and its
        // list is given out a row later, when the logits at its first entries have come.
        constexpr int kAhead = 4;                     // entries a lane asks for at a time
        Word id[kAhead];
        float ta[kAhead];
        T zk[kAhead], zlast[kAhead];
        Side side{};
        auto entries = [&](int64_t row, int k0) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (k0 + 32 * u >= a.topk) break;
                const int k = min(k0 + 32 * u + lane, a.topk - 1);
                const int64_t at = row * a.ldt + k;
                id[u] = word_at(a.ids, row * a.ldi + k);
                ta[u] = a.teacher_bf16 ? __uint_as_float(static_cast<const uint16_t*>(a.teacher)[at]) : static_cast<const float*>(a.teacher)[at];
            }
        };
        if (first < a.rows) {
            side = side_at<K>(a, first);
            entries(first, 0);
        }
        for (int64_t row = first; first < a.rows && row < a.rows + step; row += step, ++it) {
            const bool ends_here = row >= a.rows;     // only the last row's list is left
            int32_t* ids = list_of(it);
            float *qs = reinterpret_cast<float*>(ids + n1), *zs = qs + n1, *ends = zs + n1;
            const bool live = is_live<K>(a, side);
            const int32_t label = live && a.labels.p && a.hard != 0.f ? token_of<K>(a, side) : -1;
            float m = -CUDART_INF_F;
            if (!ends_here) {
                wait(smem_u32(&read_bar[it & (a.lists - 1)]), (static_cast<uint32_t>(it / a.lists) & 1u) ^ 1u, false, abort, a.err);
                const T* z = logits(row);
                auto take = [&](int k, int u) {
                    const int32_t v = live && k < a.topk ? index_of(id[u], a.ids.wide, V) : -1;
                    const float t = v < 0 ? -CUDART_INF_F : a.teacher_bf16 ? __uint_as_float(__float_as_uint(ta[u]) << 16) : ta[u];
                    if (k < a.topk) { ids[k] = v; qs[k] = t; }
                    m = fmaxf(m, t);
                    return z[max(v, 0)];
                };
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (32 * u >= a.topk) break;
                    zk[u] = take(32 * u + lane, u);
                }
#pragma unroll 1
                for (int k0 = 32 * kAhead; k0 < a.topk; k0 += 32 * kAhead) {
                    entries(row, k0);
                    T zr[kAhead];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        if (k0 + 32 * u >= a.topk) break;
                        zr[u] = take(k0 + 32 * u + lane, u);
                    }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (k0 + 32 * u + lane < a.topk) zs[k0 + 32 * u + lane] = load(&zr[u]);
                }
                const int64_t after = min(row + step, a.rows - 1);
                side = side_at<K>(a, after);
                entries(after, 0);
            }
            if (it > 0) {
                float* zs_last = reinterpret_cast<float*>(list_of(it - 1) + 2 * n1);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (32 * u + lane < a.topk) zs_last[32 * u + lane] = load(&zlast[u]);
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(smem_u32(&list_bar[(it - 1) & (a.lists - 1)]));
            }
            if (ends_here) break;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) zlast[u] = zk[u];
            m = warp_max(m);
            float sum = 0.f, tsum = 0.f;
#pragma unroll 1
            for (int k = lane; k < a.topk; k += 32) {
                const float t = qs[k];
                float w = 0.f;
                if (t != -CUDART_INF_F) {             // an entry that the teacher rules out leaves the sums as they are
                    w = exp2_fast((t - m) * c);
                    sum += w;
                    tsum += w * (t - m);
                }
                qs[k] = w;
            }
            sum = warp_sum(sum);
            tsum = warp_sum(tsum);
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll 1
            for (int k = lane; k < a.topk; k += 32) qs[k] *= inv;
            if (lane == 0) {
                ids[a.topk] = label;
                ends[0] = sum != 0.f ? 1.f : 0.f;
                ends[1] = tsum * inv * a.inv_tau - log_of(sum);
            }
        }
    } else if (warp >= nw) {
        const int sv = warp - nw;                     // rows sv, sv + 2, ..: their parity
        auto fill = [&](int64_t row, int i, const Span& sp, bool live) {      // the elected lane
            const int q = i % S;
            const uint32_t bytes = live ? static_cast<uint32_t>(sp.nv) * 16u : 0u, bar = smem_u32(&full_bar[q]);
            mbar_expect_tx(bar, bytes);
            if (bytes)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(smem_u32(slots + static_cast<size_t>(q) * a.slot_bytes)), "l"(logits(row) + sp.head + static_cast<int64_t>(sp.v0) * E),
                             "r"(bytes), "r"(bar) : "memory");
        };
        int filled = -1;                              // the last row that this warp filled a slot with
        if (sv == 0 && tc::elect_one())
            for (int q = 0; q < S; ++q)
                if (first + q * step < a.rows) { fill(first + q * step, q, row_s[q].span, row_s[q].live); filled = q; }
        // the element of the ends that this lane owns, or -1: the head with the first CTA, the tail with the last
        auto end_of = [&](const Span& sp) {
            const int tail = V - sp.head - sp.elems;
            return rank == 0 && lane < sp.head ? lane : rank == C - 1 && lane >= 8 && lane < 8 + tail ? sp.head + sp.elems + lane - 8 : -1;
        };
        // What is asked for: the teacher's entries lane and lane + 32 as they lie in memory, and two logits.
        struct Asked { Word id[2]; float a[2]; T end, zt; int e; };
        auto entry = [&](int64_t row, int k, Word& id, float& t) {
            k = min(k, a.topk - 1);
            const int64_t at = row * a.ldt + k;
            id = word_at(a.ids, row * a.ldi + k);
            t = a.teacher_bf16 ? __uint_as_float(static_cast<const uint16_t*>(a.teacher)[at]) : static_cast<const float*>(a.teacher)[at];
        };
        auto ask = [&](int64_t row, const Row& r, Asked& x) {
            const T* z = logits(row);
            x.e = end_of(r.span);
            x.end = z[max(x.e, 0)];
            x.zt = z[max(r.tok, 0)];
            if (D && FEW && a.topk > 0) {
                entry(row, lane, x.id[0], x.a[0]);
                entry(row, lane + 32, x.id[1], x.a[1]);
            }
        };
        float teach = 0.f;                            // sum of q log q of the row put down last
        bool soft_next = false;
        // ... and put down: ids, their q, their logits.  (A row is only overwritten by its gradient once all CTAs of
        // a cluster have sent its sums, which they do after this warp has met their workers' barrier.)
        auto put = [&](int64_t row, const Row& r, const Asked& x) {
            if (lane < 16) end_s[sv][lane] = x.e >= 0 ? load(&x.end) : -CUDART_INF_F;
            if (lane == 0) zt_s[sv] = load(&x.zt);
            if (!D || TEACH) return;
            if (lane == 0) id_s[sv][a.topk] = r.live && a.hard != 0.f ? r.tok : -1;
            float m = -CUDART_INF_F;
            auto take = [&](int k, const Word& word, float bits) {
                const int32_t id = r.live ? index_of(word, a.ids.wide, V) : -1;
                const float t = id < 0 ? -CUDART_INF_F : a.teacher_bf16 ? __uint_as_float(__float_as_uint(bits) << 16) : bits;
                id_s[sv][k] = id;
                q_s[sv][k] = t;
                m = fmaxf(m, t);
            };
            if (lane < a.topk) take(lane, x.id[0], x.a[0]);
            if (lane + 32 < a.topk) take(lane + 32, x.id[1], x.a[1]);
            const T* z = logits(row);
            const T z0 = z[lane < a.topk ? max(id_s[sv][lane], 0) : 0], z1 = z[lane + 32 < a.topk ? max(id_s[sv][lane + 32], 0) : 0];
            m = warp_max(m);
            float sum = 0.f, ta = 0.f;
#pragma unroll 1
            for (int k = lane; k < a.topk; k += 32) {
                const float t = q_s[sv][k];
                float w = 0.f;
                if (t != -CUDART_INF_F) {             // an entry that the teacher rules out leaves the sums as they are
                    w = exp2_fast((t - m) * c);
                    sum += w;
                    ta += w * (t - m);
                }
                q_s[sv][k] = w;
            }
            sum = warp_sum(sum);
            ta = warp_sum(ta);
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
            teach = ta * inv * a.inv_tau - log_of(sum);
            soft_next = sum != 0.f;
#pragma unroll 1
            for (int k = lane; k < a.topk; k += 32) q_s[sv][k] *= inv;
            if (lane < a.topk) z_s[sv][lane] = load(&z0);
            if (lane + 32 < a.topk) z_s[sv][lane + 32] = load(&z1);
        };
        const int64_t step2 = 2 * step;
        if (first + sv * step < a.rows) {
            Asked x;
            ask(first + sv * step, row_s[sv], x);
            put(first + sv * step, row_s[sv], x);
        }
        __syncwarp();
        it = sv;
        for (int64_t row = first + sv * step; row < a.rows; row += step2, it += 2) {
            const Row now = row_s[it & 3];
            const int top = a.topk;
            const uint32_t ph = static_cast<uint32_t>(it >> 1) & 1u;
            bool counts = now.live;
            const int32_t* ids = TEACH ? list_of(it) : id_s[sv];
            const float *qs = TEACH ? reinterpret_cast<const float*>(ids + n1) : q_s[sv], *zs = TEACH ? qs + n1 : z_s[sv];
            // (a row is only overwritten by its gradient once all CTAs of a cluster have sent its sums, which they do
            // after the barrier below: the teacher's warp has read the row's logits by then)
            if (TEACH) wait(smem_u32(&list_bar[it & (a.lists - 1)]), static_cast<uint32_t>(it / a.lists) & 1u, false, abort, a.err);
            const float tq = TEACH ? zs[n1 + 1] : teach;
            const bool soft_now = TEACH ? zs[n1] != 0.f : soft_next;
            // ---- 1
            const bool more = row + step2 < a.rows, more4 = row + 4 * step < a.rows;
            const int64_t row_f = row + S * step;
            Asked asked;
            ask(more ? row + step2 : row, row_s[(more ? it + 2 : it) & 3], asked);
            Side side{}, side_f{};
            if (tc::elect_one()) {                    // (the lane that uses them: one mask's elections agree)
                side = side_at<K>(a, more4 ? row + 4 * step : row);
                side_f = side_at<K>(a, row_f < a.rows ? row_f : row);
            }
            // ---- 2
            const int e = end_of(now.span);
            Stat st{-CUDART_INF_F, 0.f, 0.f};
            float e0 = -CUDART_INF_F;
            if (now.span.head + now.span.elems < V || now.span.head) {
                e0 = counts && lane < 16 ? end_s[sv][lane] : -CUDART_INF_F;
                if (e0 != -CUDART_INF_F) {            // exp of the one element against itself (a NaN stays one)
                    st.m = e0;
                    st.s = exp2_fast((e0 - e0) * c);
                    st.s1 = exp2_fast((e0 - e0) * kLog2e);
                }
                st = warp_merge<TWO>(st, c);
            }
            const Pub pub{counts ? zt_s[sv] : 0.f, D && counts && soft_now};
            if (lane == 0) {
                stat_s[sv][nw] = st;
                pub_s[sv] = pub;
                if (C > 1) mbar_expect_tx(smem_u32(&x_bar[sv]), 16u * C);
            }
            __syncwarp();
            if (sv) asm volatile("bar.arrive 2, %0;" ::"r"(nt + 32) : "memory");
            else asm volatile("bar.arrive 1, %0;" ::"r"(nt + 32) : "memory");
            // ---- 3
            wait(smem_u32(&fin_bar[sv]), ph, false, abort, a.err);
            st = fin_s[sv];
            if (st.s == 0.f) counts = false;
            const Coef k = coef_of<K, TWO>(a, now, st, pub, counts);
            if (D) {
                const bool soft = counts && pub.soft && a.soft != 0.f;    // (the divergence may be infinite)
                float zq = 0.f;
                if (soft) {
#pragma unroll 1
                    for (int j = lane; j < top; j += 32) {
                        const float w = qs[j];
                        if (w != 0.f) zq += w * (zs[j] - st.m);
                    }
                    zq = warp_sum(zq);
                }
                if (lane == 0 && rank == 0) {
                    float loss = 0.f;
                    if (soft) loss = a.soft * (tq - (zq * a.inv_tau - log_of(st.s)));
                    if (counts && now.tok >= 0 && a.hard != 0.f) loss += a.hard * (log_of(st.s1) - (pub.zt - st.m));
                    a.row_loss[row] = loss;
                }
            } else if (lane == 0 && rank == 0) {
                a.logp[row] = k.lp;
                if (K == kPolicy) {
                    a.row_loss[row] = k.loss;
                } else {
                    a.sums[row] = RowSum{st.m, counts ? log2f(st.s) : CUDART_INF_F, 0.f, 0.f};
                }
            }
            // ---- 4
            wait(smem_u32(&dense_bar[sv]), ph, false, abort, a.err);
            if (grad) {
                uint8_t* slot = slots + static_cast<size_t>(it % S) * a.slot_bytes;
                T* body = gradient(row) + now.span.head + static_cast<int64_t>(now.span.v0) * E;
                T* mine = now.same ? reinterpret_cast<T*>(slot) : body;
                auto at = [&](float x) {
                    const float d = x - st.m;
                    float g = k.dense * exp2_fast(d * c);
                    if (TWO) g += k.dense1 * exp2_fast(d * kLog2e);
                    return g;
                };
                // where an id lies: its place in this CTA's part of the row; -2 - i: the end i that this CTA owns; -1: elsewhere
                auto place = [&](int32_t v) {
                    const int b = v - now.span.head - now.span.v0 * E;
                    if (v < now.span.head) return rank == 0 ? -2 - v : -1;
                    if (v >= now.span.head + now.span.elems) return rank == C - 1 ? -10 - (v - now.span.head - now.span.elems) : -1;
                    return b < now.span.nv * E ? max(b, -1) : -1;
                };
                if (e >= 0) store(gradient(row) + e, counts ? at(e0) : 0.f);
                __syncwarp();
                if (!D && counts && lane == 0) {
                    const int b = place(now.tok);
                    if (b != -1) store(b >= 0 ? mine + b : gradient(row) + now.tok, at(pub.zt) - k.at_tok);
                }
                if (D && counts) {
                    // Entries mark their places in the slot (or an end's) with their number.  One that finds another's
                    // mark there shares its id: it flags the mark, and the flagged mark's owner adds up all of that id.
                    using M = typename Vec<T>::Mark;
                    constexpr int kFlag = 1 << 14;
                    const float f = now.w * a.soft * a.inv_tau;
                    M* marks = reinterpret_cast<M*>(slot);
                    auto value = [&](int j) { return j < top ? (pub.soft ? f * qs[j] : 0.f) : k.at_tok; };
                    const int n = ids[top] >= 0 ? top + 1 : top;
#pragma unroll 1
                    for (int j = lane; j < n; j += 32) {
                        const int b = ids[j] >= 0 ? place(ids[j]) : -1;
                        if (b >= 0) marks[b] = static_cast<M>(j);
                        else if (b != -1) mark_s[sv][-2 - b] = j;
                    }
                    __syncwarp();
                    uint64_t lost = 0;                // bit u: entry lane + 32 u found another's mark
#pragma unroll 1
                    for (int j = lane; j < n; j += 32) {
                        const int b = ids[j] >= 0 ? place(ids[j]) : -1;
                        const int r = b >= 0 ? static_cast<int>(marks[b]) : b != -1 ? mark_s[sv][-2 - b] : j;
                        if ((r & (kFlag - 1)) != j) {
                            lost |= uint64_t(1) << (j >> 5);
                            if (b >= 0) marks[b] = static_cast<M>(r | kFlag);
                            else mark_s[sv][-2 - b] = r | kFlag;
                        }
                    }
                    const bool twice = __any_sync(~0u, lost != 0);
                    __syncwarp();
#pragma unroll 1
                    for (int j = lane; j < n; j += 32) {
                        const int32_t v = ids[j];
                        const int b = v >= 0 ? place(v) : -1;
                        if (b == -1) continue;
                        float g = value(j);
                        if (twice) {
                            if (lost >> (j >> 5) & 1) continue;
                            const int r = b >= 0 ? static_cast<int>(marks[b]) : mark_s[sv][-2 - b];
                            if (r & kFlag) {
                                g = 0.f;
#pragma unroll 1
                                for (int i = 0; i < n; ++i) g += ids[i] == v ? value(i) : 0.f;
                            }
                        }
                        store(b >= 0 ? mine + b : gradient(row) + v, at(j < top ? zs[j] : pub.zt) - g);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // the workers' writes and these, before the copy reads them
                __syncwarp();
                if (tc::elect_one()) {
                    if (now.span.nv > 0 && now.same)
                        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                                     ::"l"(body), "r"(smem_u32(slot)), "r"(static_cast<uint32_t>(now.span.nv) * 16u) : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            }
            __syncwarp();
            // ---- 5, and the slot's next row once it has been read
            if (more) put(row + step2, row_s[(it + 2) & 3], asked);
            if (tc::elect_one()) {
                if (TEACH) tc::mbar_arrive(smem_u32(&read_bar[it & (a.lists - 1)]));
                if (row_f < a.rows) {
                    if (grad) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    fill(row_f, it + S, span_of(logits(row_f), V, rank, a.cluster_shift), is_live<K>(a, side_f));
                    filled = it + S;
                }
                if (more4) prepare(row + 4 * step, it + 4, side);
            }
            __syncwarp();
        }
        if (tc::elect_one()) {
            if (grad) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            if (*abort)                               // let the copies that this warp issued land
                for (int i = max(filled - 3, 0); i <= filled; ++i)
                    for (int q = 0; q < 1000000 && !try_wait(smem_u32(&full_bar[i % S]), static_cast<uint32_t>(i / S) & 1u, false); ++q) __nanosleep(64);
        }
    } else {
        for (int64_t row = first; row < a.rows; row += step, ++it) {
            const int par = it & 1;
            const Row now = row_s[it & 3];
            const int nv = now.span.nv;
            bool counts = now.live;
            uint4* slot = reinterpret_cast<uint4*>(slots + static_cast<size_t>(s) * a.slot_bytes);
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
                        if (TWO) t2[i & 1] = TWO >= kSquares ? power_sum<TWO>(e, t2[i & 1]) : add2(t2[i & 1], exp2_2(mul2(d, l2)));
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
                        const uint64_t d = add2(x[i], nr), e = exp2_2(mul2(d, c2));
                        s2 = add2(s2, e);
                        if (TWO) t2 = TWO >= kSquares ? power_sum<TWO>(e, t2) : add2(t2, exp2_2(mul2(d, l2)));
                    }
                }
                float x, y;
                unpack2(s2, x, y);
                st.s = x + y;
                unpack2(t2, x, y);
                st.s1 = x + y;
            }
            const float m_own = st.m;                 // what this thread's exponentials are relative to
            st = warp_merge<TWO>(st, c);
            if (lane == 0) stat_s[par][warp] = st;
            __syncwarp();
            if (par) asm volatile("bar.sync 2, %0;" ::"r"(nt + 32) : "memory");
            else asm volatile("bar.sync 1, %0;" ::"r"(nt + 32) : "memory");
            st = warp_merge<TWO>(lane <= nw ? stat_s[par][lane] : Stat{-CUDART_INF_F, 0.f, 0.f}, c);
            const Pub pub = pub_s[par];
            if (C > 1) {
                // the sums go to the peers with the signal that they are there, in one store each
                if (warp == 0 && lane < C)
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                                 ::"r"(peer_addr(smem_u32(&cluster_s[par][rank]), lane)), "f"(st.m), "f"(st.s), "f"(st.s1), "f"(0.f),
                                   "r"(peer_addr(smem_u32(&x_bar[par]), lane)) : "memory");
                wait(smem_u32(&x_bar[par]), xuse, true, abort, a.err);
                const float4 x = lane < C ? cluster_s[par][lane] : make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
                st = warp_merge<TWO>(Stat{x.x, x.y, x.z}, c);
            }
            if (!TWO) st.s1 = st.s;
            if (tid == 0) {
                fin_s[par] = st;
                tc::mbar_arrive(smem_u32(&fin_bar[par]));
            }
            if (st.s == 0.f) counts = false;
            // ---- the gradient
            if (grad) {
                const Coef k = coef_of<K, TWO>(a, now, st, pub, counts);
                const uint64_t nm = pack2(-st.m, -st.m), dd1 = pack2(k.dense1, k.dense1);
                T* body = gradient(row) + now.span.head + static_cast<int64_t>(now.span.v0) * E;
                auto put = [&](int v, const uint4& u) {
                    if (now.same) slot[v] = u;
                    else Vec<T>::scatter(body + v * E, u);     // the gradient's rows lie otherwise on 16 bytes
                };
                if (counts && HELD) {
                    const float f = k.dense * shrink(m_own, st.m, c);
                    const uint64_t ff = pack2(f, f);
                    const float f1 = TWO >= kSquares ? k.dense1 * shrink(m_own, st.m, kLog2e) : 0.f;
                    const uint64_t ff1 = pack2(f1, f1);
#pragma unroll
                    for (int j = 0; j < kKeep; ++j) {
                        const int v = tid + j * nt;
                        if (v < nv) {
                            uint64_t x[P];
                            if (TWO == kBoth) Vec<T>::get(slot[v], x);
#pragma unroll
                            for (int i = 0; i < P; ++i) {
                                const uint64_t e = kept[j][i], g = mul2(ff, e);
                                x[i] = TWO == kBoth ? fma2(dd1, exp2_2(mul2(add2(x[i], nm), l2)), g)
                                     : TWO >= kSquares ? two_powers<TWO>(ff, ff1, e) : g;
                            }
                            put(v, Vec<T>::put(x));
                        }
                    }
                } else if (counts) {
                    const uint64_t dd = pack2(k.dense, k.dense);
                    for (int v = tid; v < nv; v += nt) {
                        uint64_t x[P];
                        Vec<T>::get(slot[v], x);
#pragma unroll
                        for (int i = 0; i < P; ++i) {
                            const uint64_t d = add2(x[i], nm), e = exp2_2(mul2(d, c2));
                            x[i] = TWO == kBoth ? fma2(dd1, exp2_2(mul2(d, l2)), mul2(dd, e)) : TWO >= kSquares ? two_powers<TWO>(dd, dd1, e) : mul2(dd, e);
                        }
                        put(v, Vec<T>::put(x));
                    }
                } else {
                    for (int v = tid; v < nv; v += nt) put(v, make_uint4(0, 0, 0, 0));
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(smem_u32(&dense_bar[par]));
            if (++s == S) { s = 0; use ^= 1u; }
            if (par) xuse ^= 1u;
        }
    }
    // no CTA of a cluster leaves while another may still write to its shared memory
    if (C > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

constexpr int kThreads = 256;

// Sums as pairs of floats, the second one the rounding errors of the first (64-bit arithmetic runs at a
// hundredth of the rate here): thread by thread, then up a tree, in a fixed order.
struct Pair { float hi, lo; };
__device__ __forceinline__ Pair plus(const Pair& x, const Pair& y) {
    const float s = x.hi + y.hi, b = s - x.hi, err = (x.hi - (s - b)) + (y.hi - b);
    return {s, isfinite(s) ? err + x.lo + y.lo : 0.f};
}
__device__ Pair block_sum(Pair x, Pair* scratch) {
    for (int d = 16; d; d >>= 1) x = plus(x, Pair{__shfl_xor_sync(~0u, x.hi, d), __shfl_xor_sync(~0u, x.lo, d)});
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    x = lane < static_cast<int>(blockDim.x >> 5) ? scratch[lane] : Pair{0.f, 0.f};
    for (int d = 16; d; d >>= 1) x = plus(x, Pair{__shfl_xor_sync(~0u, x.hi, d), __shfl_xor_sync(~0u, x.lo, d)});
    return x;
}

constexpr int kPairThreads = 256;
// One CTA a pair.
__global__ void __launch_bounds__(kPairThreads) pairs_kernel(const PairArgs a) {
    chain_begin();
    __shared__ Pair scratch[kPairThreads / 32];
    const int64_t p = blockIdx.x;
    int64_t at[2][2];
    float seq[2], share[2];
    for (int h = 0; h < 2; ++h) {
        int64_t b = a.offsets.at(2 * p + h), e = a.offsets.at(2 * p + h + 1);
        b = b < 0 ? 0 : b > a.rows ? a.rows : b;
        e = e < b ? b : e > a.rows ? a.rows : e;
        at[h][0] = b; at[h][1] = e;
        Pair sum{0.f, 0.f};
        int cnt = 0;
        for (int64_t t = b + threadIdx.x; t < e; t += kPairThreads) {
            sum = plus(sum, Pair{a.row_logp[t], 0.f});
            cnt += a.sums[t].log2_sum != CUDART_INF_F;
        }
        sum = block_sum(sum, scratch);
        share[h] = 1.f;
        seq[h] = sum.hi + sum.lo;
        if (a.average) {
            // (the number of tokens, exactly: its two halves as floats)
            const Pair n = block_sum(Pair{static_cast<float>(cnt), 0.f}, scratch);
            share[h] = 1.f / fmaxf(n.hi + n.lo, 1.f);
            seq[h] = seq[h] / fmaxf(n.hi + n.lo, 1.f);
        }
    }
    const float w = a.weight ? a.weight[p] : a.share;
    const float h = (seq[0] - (a.ref_logp ? a.ref_logp[2 * p] : 0.f)) - (seq[1] - (a.ref_logp ? a.ref_logp[2 * p + 1] : 0.f));
    float loss, slope;
    if (a.kind == GLR_PREF_IPO) {
        const float e = h - 0.5f / a.beta;
        loss = e * e;
        slope = 2.f * e;
    } else {
        // -log sigmoid(x) = max(-x, 0) + log1p(exp(-|x|)); a term whose share is 0 is left out: it may be infinite
        const float x = a.beta * h, t = log1pf(expf(-fabsf(x)));
        loss = 0.f;
        if (a.smoothing != 1.f) loss = (1.f - a.smoothing) * (fmaxf(-x, 0.f) + t);
        if (a.smoothing != 0.f) loss += a.smoothing * (fmaxf(x, 0.f) + t);
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
            if (a.sums[t].log2_sum != CUDART_INF_F) a.sums[t].coef = coef;
    }
}

// Sixteen bytes past the caches' keeping: the second and last read of a row, and its gradient.
__device__ __forceinline__ uint4 load_last(const void* p) {
    uint4 u;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}
__device__ __forceinline__ void store_last(void* p, const uint4& u) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
}

// dz = coef (e_token - exp2((z - m) log2 e - log2 s)): the second pass over a preference batch's rows (its factor needs the
// whole pair first), a piece of a row a CTA.  m and log2 s come apart from the first pass: their sum would lose the
// latter beside an m of 1e5, and all of it at the type's lowest value.  Rows are taken from the last one back: the sums'
// pass ended there, and the L2 still holds some 100 MB of it.  Bound by HBM: one read, one write (8 pairs of 2 x 512 rows
// of 32768 bf16: 249 us with the sums' pass, 4.3 TB/s of one read and one write, 6.5 of the two reads that it makes).
constexpr int kPieceVecs = 4;
template <class T>
__global__ void __launch_bounds__(kThreads) grad_kernel(const RowArgs a, int pieces) {
    chain_begin();
    constexpr int E = Vec<T>::kElems, P = E / 2;
    const int64_t row = a.rows - 1 - blockIdx.x / pieces;
    const int piece = static_cast<int>(blockIdx.x % pieces), V = static_cast<int>(a.vocab), tid = threadIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.ldz;
    T* dz = static_cast<T*>(a.dz) + row * a.lddz;
    const RowSum sum = a.sums[row];
    const float coef = sum.coef, m = sum.top, ls = sum.log2_sum;
    const int32_t tok = index_of(word_at(a.tokens, row), a.tokens.wide, V);
    const bool zero = coef == 0.f;
    auto at = [&](float x, int v) {
        const float g = -coef * exp2_fast(fmaf(x - m, kLog2e, -ls));
        return v == tok ? g + coef : g;
    };
    const Span sp = span_of(z, V, 0, 0);
    if (piece == 0) {                                 // the unaligned ends
        const int v = tid < sp.head ? tid : tid >= 32 && tid < 32 + V - sp.head - sp.elems ? sp.head + sp.elems + tid - 32 : -1;
        if (v >= 0) store(dz + v, zero ? 0.f : at(load(z + v), v));
    }
    const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
    const int v0 = piece * (kThreads * kPieceVecs) + tid;
    uint4 u[kPieceVecs];
    if (!zero) {
#pragma unroll
        for (int q = 0; q < kPieceVecs; ++q)
            if (v0 + q * kThreads < sp.nv) u[q] = load_last(z + sp.head + static_cast<int64_t>(v0 + q * kThreads) * E);
    }
    const uint64_t nm = pack2(-m, -m), nl = pack2(-ls, -ls), l2 = pack2(kLog2e, kLog2e), nc = pack2(-coef, -coef);
#pragma unroll
    for (int q = 0; q < kPieceVecs; ++q) {
        const int v = v0 + q * kThreads, b = tok - sp.head - v * E;
        if (v >= sp.nv) break;
        uint4 r = make_uint4(0, 0, 0, 0);
        if (!zero) {
            uint64_t x[P];
            Vec<T>::get(u[q], x);
#pragma unroll
            for (int i = 0; i < P; ++i) x[i] = mul2(nc, exp2_2(fma2(add2(x[i], nm), l2, nl)));
            if (tok >= 0 && b >= 0 && b < E) {
#pragma unroll
                for (int i = 0; i < P; ++i) x[i] = add2(x[i], pack2(b == 2 * i ? coef : 0.f, b == 2 * i + 1 ? coef : 0.f));
            }
            r = Vec<T>::put(x);
        }
        T* to = dz + sp.head + static_cast<int64_t>(v) * E;
        if (same) store_last(to, r);
        else Vec<T>::scatter(to, r);
    }
}

constexpr int kTotalThreads = 1024;
__global__ void __launch_bounds__(kTotalThreads) total_kernel(const float* x, const float* weight, float share, int64_t n,
                                                              float* out) {
    chain_begin();
    __shared__ Pair scratch[kTotalThreads / 32];
    Pair s{0.f, 0.f};
    for (int64_t i = threadIdx.x; i < n; i += kTotalThreads) {
        const float w = weight ? weight[i] : share, v = x[i];
        if (w != 0.f) {
            const float p = w * v;
            s = plus(s, Pair{p, isfinite(p) ? fmaf(w, v, -p) : 0.f});
        }
    }
    s = block_sum(s, scratch);
    if (threadIdx.x == 0) *out = s.hi + s.lo;
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
    const bool few = K != kDistill || a.topk <= kFewEntries;
    const int most = most_workers(few);
    while (C < kMaxCluster && (vecs + C - 1) / C * 16 > slot_max(most)) C *= 2;
    // few rows: more CTAs a row, as long as each has 4 KiB of it (one row of 131072 bf16 15 -> 13 us, 33 of 32768 14 -> 13,
    // each with the total's launch)
    while (C < kMaxCluster && a.rows * C * 2 <= sms && row_bytes / (2 * C) >= 4096) C *= 2;
    a.cluster_shift = C == 1 ? 0 : C == 2 ? 1 : C == 4 ? 2 : 3;
    a.slot_bytes = static_cast<uint32_t>((vecs + C - 1) / C * 16);
    // the teacher's lists: four, or two beside the longest slots
    const int64_t list = few ? 0 : 4 * list_words(a.topk);
    a.lists = kMaxLists;
    if (a.lists * list + a.slot_bytes > kDynMax) a.lists = 2;
    a.slots = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(3, std::min(kRingMax, kDynMax - a.lists * list) / a.slot_bytes)));
    const size_t smem = static_cast<size_t>(a.slots) * a.slot_bytes + a.lists * list;
    const bool held = a.slot_bytes <= slot_max(most);
    const int workers = held ? static_cast<int>((a.slot_bytes / 16 + 32 * kHeld - 1) / (32 * kHeld)) : most, extra = few ? 2 : 3;
    const int two = K != kDistill || !a.labels.p || a.hard == 0.f || a.inv_tau == 1.f ? 0 : a.inv_tau == 0.5f ? kSquares : a.inv_tau == 0.25f ? kFourths : kBoth;
    auto pick = [&](auto t) {
        using T = decltype(t);
        constexpr bool D = K == kDistill;
        auto of = [&](auto few_entries, auto held_slots) {
            constexpr bool F = decltype(few_entries)::value || !D, H = decltype(held_slots)::value;
            return two == kBoth ? rows_kernel<K, T, H, D ? kBoth : 0, F>
                 : two == kSquares ? rows_kernel<K, T, H, D ? kSquares : 0, F>
                 : two == kFourths ? rows_kernel<K, T, H, D ? kFourths : 0, F> : rows_kernel<K, T, H, 0, F>;
        };
        return few ? (held ? of(std::true_type(), std::true_type()) : of(std::true_type(), std::false_type()))
                   : (held ? of(std::false_type(), std::true_type()) : of(std::false_type(), std::false_type()));
    };
    auto kernel = dtype == GLR_BF16 ? pick(__nv_bfloat16()) : pick(float());
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kDynMax))) != cudaSuccess) return e;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = C; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = (workers + extra) * 32; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    // as many groups of CTAs as run at once, each with its share of the rows
    int64_t groups = a.rows;
    if (a.rows * C > sms) {
        int per = 0;
        cfg.gridDim = C;
        if (C > 1) e = cudaOccupancyMaxActiveClusters(&per, kernel, &cfg);
        else if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, (workers + extra) * 32, smem)) == cudaSuccess) per *= sms;
        if (e != cudaSuccess) return e;
        groups = std::min<int64_t>(groups, std::max(per, 1));
    }
    cfg.gridDim = static_cast<unsigned>(groups * C);
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
    const int64_t vecs = a.vocab * (dtype == GLR_BF16 ? 2 : 4) / 16, per = kThreads * kPieceVecs;
    const int pieces = static_cast<int>(std::max<int64_t>(1, (vecs + per - 1) / per));
    const unsigned grid = static_cast<unsigned>(a.rows * pieces);
    return dtype == GLR_BF16 ? launch_chain(grad_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, pieces)
                             : launch_chain(grad_kernel<float>, grid, kThreads, 0, st, a, pieces);
}

cudaError_t total(const float* x, const float* weight, float share, int64_t n, float* out, cudaStream_t st) {
    return launch_chain(total_kernel, 1, kTotalThreads, 0, st, x, weight, share, n, out);
}

}  // namespace loss
}  // namespace glr
