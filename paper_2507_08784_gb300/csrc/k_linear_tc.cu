// Products of linear layers on the fifth-generation tensor cores: out = epilogue(A B^T) for bf16 operands
// whose rows lie on 16 bytes, either operand contiguous along the contraction ("K-major") or along its own
// index ("MN-major"), so that the forward product, the input's gradient and the weights' gradients all read
// their matrices as they are.  Matrices that lie otherwise are copied into rows on 16 bytes first, and fp32
// ones into three bf16 planes x = hi + mid + lo (24 bits; below 2^-110 the lower ones leave bf16's range): their product
// is the sum of the six plane products above 2^-24, one after the other in the same accumulator.
//
// tc_product_kernel, persistent: a pair of CTAs on two SMs takes 256 x 256 output tiles in turn.  Two warps of each copy
// operand slabs of 64 contraction elements (128-byte swizzle) into a ring of shared-memory stages, one thread of the
// pair's first CTA issues tcgen05.mma.kind::f16 (each CTA holds its 128 rows of A and half of B's, and the result's rows
// stay in their CTA's tensor memory), and eight warps (sixteen for fp32 results) bring the finished accumulator through the
// epilogue while the next tile's products run into the other half of tensor memory.  Stages are handed over on mbarriers;
// every wait is bounded: a CTA that gives up counts the event, lets its copies land, frees tensor memory and returns.
// tc_split_kernel, for few tiles: a cluster of up to eight CTAs shares a 128 x 64 tile's contraction (CG = 1), or two pairs
// a 256 x 256 one's (CG = 2), and they add their partial tiles over distributed shared memory in the order of the
// contraction.
//
// The tensor cores truncate their fp32 sums, always the same way: 2^-25 of the sum for every 16 elements, or more, which
// over a long contraction is far above fp32 rounding.  Where the result is fp32, and in tc_split_kernel, the sums of 256
// contraction elements (64 of three planes) join the total in rounded additions by the epilogue warps (PROMOTE); where
// it is bf16, whole tiles' sums are truncated throughout up to kMostTruncated elements, and promoted every 4096 (1024) beyond.
//
// What bounds it: the tensor pipe for contractions of about 1000 and more, 512 cycles a 256 x 256 x 64 stage (8192 x
// 11008 x 4096 bf16 with SiLU and pre-activation: 467 us among other passes, 1.58 PFLOP/s under the power cap; 408 in a
// short row of calls, at a higher clock); below that the epilogue (8192 x 2048 x 512: 28 us); for few tiles the loads'
// latency; with sums promoted every 256 elements also the reads of tensor memory, a chunk's in about the time of its
// products, and the sums' way back through it at the end (5632 x 2048 of eight nodes' 1024 rows: 113 us to bf16, 207 to
// fp32).  fp32: six products a slab, 4096 x 4096 x 2048 332 to 350 us.  Tensor memory gives a thread a row; the epilogue
// warps turn 32 x 32 blocks round in shared memory, so that four lanes share a row and an access covers whole sectors
// of eight rows.
#include <algorithm>

#include "glr_host.cuh"
#include "glr_linear.cuh"
#include "glr_ptx.cuh"

namespace glr {
namespace linear {

namespace {

using tc::elect_one;
using tc::fence_after;
using tc::fence_before;
using tc::mbar_expect_tx;
using tc::mbar_init;
using tc::smem_u32;

constexpr int epi_warps(bool promote) { return promote ? 16 : 8; }     // ... of 64 or 128 columns each
constexpr int threads_of(int epi) { return (epi + 3) * 32; }             // ... and two copying warps and the issuer
constexpr int kSlab = 64;                       // contraction elements a stage: one 128-byte swizzle row of bf16
constexpr int kMaxStages = 8;
constexpr size_t kSmemBytes = 224 * 1024;       // of it the ring has what the epilogue warps' blocks leave
constexpr int kBlockPitch = 36;                 // floats a row of a 32 x 32 block: no two lanes on a bank
constexpr size_t kBlockBytes = 32 * kBlockPitch * 4;
constexpr int kBand = 8;                        // tile rows walked together, so that a wave's operands share L2

struct TcArgs {
    Product p;
    CUtensorMap mapA, mapB;
    int tiles_m, tiles_n, slabs, stages;
    int tiles, whole;                           // tiles in all; from `whole` on they are halves of BN / 2 columns
    int planes;                                 // 1, or 3: a slab of the contraction is six products of planes
    int chunk;                                  // slabs whose sums are kept in tensor memory (PROMOTE)
    int wide;                                   // 16-byte accesses: bit 0 out, 1 bias, 2 add, 3 pre, 4 aux
    int columns;                                // some of them but the bias not: epilogues take columns
};

template <int BN, int CG>
constexpr uint32_t stage_bytes() { return 128 * 128 + BN / CG * 128; }

__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// (What these barriers hand over is read by tile copies, MMAs and tensor-memory loads, which their commits and
// the tcgen05 fences order.  A wait that acquires for the cluster would clear the L1 each time, and an arrival
// that releases for it would wait for the stores before it: together 690 cycles for the issuer's 512-cycle slab.)
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Bounded wait for a phase; false once the CTA has given up.  The first polls follow each other at once (a
// slab's products take a quarter of a microsecond), the later ones sleep, for about a second.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort, int* err) {
    for (int it = 0; it < 16000000; ++it) {
        if (try_wait(bar, parity)) return true;
        if (it >= 64) {
            if ((it & 63) == 0 && *abort) return false;
            __nanosleep(64);
        }
    }
    if (atomicExch(const_cast<int*>(abort), 1) == 0) atomicAdd(err, 1);
    return false;
}
template <int CG>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory matrix descriptors of the 128-byte swizzle.  K-major: 8-row groups 1024 bytes apart.
// MN-major: 64-element chunks of the operand's index `chunk` bytes apart, 8-slab-row groups 1024.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn, uint32_t chunk) {
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(mn ? chunk >> 4 : 1) << 16) |
           (uint64_t(64) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
    if (CG == 1)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(acc));
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(acc));
}
// Arrives on `bar` (of the CTAs of `mask`) when the products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar, uint16_t mask = 1) {
    if (CG == 1) tc::mma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(mask) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t ta, float (&v)[32]) {
    uint32_t u[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
                   "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]),
                   "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]),
                   "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
                 : "r"(ta));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
}

// sum += sixteen columns (what 32 at a time would take beside the sums does not fit the registers).
__device__ __forceinline__ void tmem_add16(uint32_t ta, float* sum) {
    uint32_t u[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
                   "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(ta));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[j] += __uint_as_float(u[j]);
}
__device__ __forceinline__ void tmem_store32(uint32_t ta, const float* v) {
    uint32_t u[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(v[j]);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
                   "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]),
                   "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]),
                   "r"(u[30]), "r"(u[31]), "r"(ta) : "memory");
}

// Eight elements at p, `step` apart (n of them in range; wide: neighbours, on 16 bytes), widened.
__device__ __forceinline__ void widen8(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v[2 * q] = __uint_as_float(w[q] << 16);
        v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
    }
}
__device__ __forceinline__ void get8(const void* base, int64_t at, int n, bool wide, int dtype, float (&v)[8], int64_t step = 1) {
    if (dtype == GLR_F32) {
        const float* p = static_cast<const float*>(base) + at;
        if (wide && n == 8) {
            const float4 x = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e * step] : 0.f;
        }
        return;
    }
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + at;
    if (wide && n == 8) {
        widen8(*reinterpret_cast<const uint4*>(p), v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? __bfloat162float(p[e * step]) : 0.f;
    }
}
__device__ __forceinline__ void put8(void* base, int64_t at, int n, bool wide, int dtype, const float (&v)[8], int64_t step = 1) {
    if (dtype == GLR_F32) {
        float* p = static_cast<float*>(base) + at;
        if (wide && n == 8) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (e < n) p[e * step] = v[e];
        }
        return;
    }
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + at;
    if (wide && n == 8) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * q], v[2 * q + 1]);
            w[q] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < n) p[e * step] = __float2bfloat16_rn(v[e]);
    }
}
template <bool SLOPE, bool FAST>
__device__ __forceinline__ void act8(float (&v)[8], int act) {
    switch (act) {                               // one branch for the eight
#define GLR_ACT_CASE(A)                                                                               \
        case A:                                                                                       \
            _Pragma("unroll") for (int e = 0; e < 8; ++e) v[e] = SLOPE ? act_slope<FAST>(v[e], A) : act_value<FAST>(v[e], A); \
            break;
        GLR_ACT_CASE(GLR_ACT_RELU)
        GLR_ACT_CASE(GLR_ACT_GELU)
        GLR_ACT_CASE(GLR_ACT_GELU_TANH)
        GLR_ACT_CASE(GLR_ACT_SILU)
#undef GLR_ACT_CASE
        default: break;
    }
}

// The epilogue on eight elements: acc in v.  They are neighbouring columns of a row (i, j), or with COLUMN neighbouring
// rows of a column, for matrices that do not lie on 16 bytes: then neighbouring lanes are neighbouring columns, and an
// access covers whole sectors all the same (4096 x 4096 x 512 bf16, results in rows of 4099: 83 -> 40 us).
// add and pre, unless null: the row's eight elements of either, asked for earlier.
template <int MODE, int DT, bool COLUMN>
__device__ __forceinline__ void epilogue8(const TcArgs& a, int node, int64_t i, int64_t j, float (&v)[8], const uint4* add = nullptr,
                                          const uint4* pre = nullptr) {
    const Product& p = a.p;
    constexpr int dt = DT;                      // of the results, and but in kGradWeight of the inputs too
    const int64_t left = COLUMN ? p.M - i : p.N - j;
    const int n = static_cast<int>(left < 8 ? left : 8);
    auto get = [&](const void* x, int64_t ld, int bit, float (&f)[8]) { get8(x, i * ld + j, n, !COLUMN && (a.wide & bit), dt, f, COLUMN ? ld : 1); };
    auto put = [&](void* x, int64_t ld, int bit, const float (&f)[8]) { put8(x, i * ld + j, n, !COLUMN && (a.wide & bit), dt, f, COLUMN ? ld : 1); };
    auto added = [&](const float (&f)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += f[e];
    };
    if (MODE == kGradWeight) {
        put(p.outs[node], p.N, 1, v);
        return;
    }
    float x[8];
    if (p.add) {
        if (add && n == 8) widen8(*add, x);
        else get(p.add, p.ldadd, 4, x);
    }
    if (MODE == kForward) {
        if (p.bias) {
            float b[8];
            get8(p.bias, j, COLUMN ? 8 : n, !COLUMN && (a.wide & 2), dt, b, COLUMN ? 0 : 1);
            added(b);
        }
        if (p.aux) put(p.aux, p.ldaux, 16, v);
        act8<false, DT == GLR_BF16>(v, p.act);
        if (p.add) added(x);
    } else {
        if (p.add) added(x);
        if (p.aux) put(p.aux, p.ldaux, 16, v);
        if (p.pre) {
            if (pre && n == 8) widen8(*pre, x);
            else get(p.pre, p.ldpre, 8, x);
            act8<true, DT == GLR_BF16>(x, p.act);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= x[e];
        }
    }
    put(p.out, p.ldo, 1, v);
}

struct Tile { int node, m, n0, bn; };
template <int BN>
__device__ __forceinline__ Tile tile_at(const TcArgs& a, int t) {
    Tile r;
    r.bn = BN;
    int half = 0;
    if (t >= a.whole) {                              // the last ones as halves, for twice as many CTAs
        half = (t - a.whole) & 1;
        t = a.whole + ((t - a.whole) >> 1);
        r.bn = BN / 2;
    }
    const int per = a.tiles_m * a.tiles_n;
    r.node = t / per;
    t -= r.node * per;
    const int band = t / (kBand * a.tiles_n), in = t - band * kBand * a.tiles_n;
    const int h = min(kBand, a.tiles_m - band * kBand);
    r.m = band * kBand + in % h;
    r.n0 = in / h * BN + half * (BN / 2);
    return r;
}

// The planes of A and B in the six products of a slab, the smallest first.
__device__ __forceinline__ int plane_a(int pair) { return pair == 0 ? 2 : pair == 2 || pair == 3 ? 1 : 0; }
__device__ __forceinline__ int plane_b(int pair) { return pair == 1 ? 2 : pair == 2 || pair == 4 ? 1 : 0; }

// The tile copies of stage k (slab k, or product k mod 6 of slab k / 6): rows m0.. of A, and `nb` 64-row pieces of B
// from n0 on.
template <int CG, bool MNA, bool PLANES>
__device__ __forceinline__ void load_a(const TcArgs& a, int k, int m0, int node, uint32_t st, uint32_t bar) {
    int x = k * kSlab, z = node;
    if (PLANES && a.planes == 3) {
        const int slab = k / 6;
        x = slab * kSlab;
        z += a.p.nodes * plane_a(k - 6 * slab);
    }
    if (MNA) {
        load_3d<CG>(st, &a.mapA, m0, x, z, bar);
        load_3d<CG>(st + 8192, &a.mapA, m0 + 64, x, z, bar);
    } else {
        load_3d<CG>(st, &a.mapA, x, m0, z, bar);
    }
}
template <int CG, bool MNB, bool PLANES>
__device__ __forceinline__ void load_b(const TcArgs& a, int k, int n0, int nb, int node, uint32_t st, uint32_t bar) {
    int x = k * kSlab, z = node;
    if (PLANES && a.planes == 3) {
        const int slab = k / 6;
        x = slab * kSlab;
        z += a.p.nodes * plane_b(k - 6 * slab);
    }
    for (int c = 0; c < nb; ++c) {
        if (MNB) load_3d<CG>(st + 16384 + c * 8192, &a.mapB, n0 + 64 * c, x, z, bar);
        else load_3d<CG>(st + 16384 + c * 8192, &a.mapB, x, n0 + 64 * c, z, bar);
    }
}
// ... and its MMAs, sixteen contraction elements each, on `bn` columns.
template <int CG, bool MNA, bool MNB>
__device__ __forceinline__ void mma_stage(uint32_t d, uint32_t st, int bn, bool add) {
    const uint32_t id = (1u << 4) | (1u << 7) | (1u << 10) | (MNA ? 1u << 15 : 0u) | (MNB ? 1u << 16 : 0u) |
                        (static_cast<uint32_t>(bn >> 3) << 17) | (static_cast<uint32_t>(8 * CG) << 24);
#pragma unroll
    for (int kk = 0; kk < kSlab / 16; ++kk)
        mma_f16<CG>(d, operand_desc(st + (MNA ? 2048 : 32) * kk, MNA, 8192),
                    operand_desc(st + 16384 + (MNB ? 2048 : 32) * kk, MNB, 8192), id, (add || kk) ? 1u : 0u);
}

// A warp's columns of an accumulator have been read: its barrier, of the pair's first CTA `lead`.
template <int CG>
__device__ __forceinline__ void hand_back(uint32_t bar, uint32_t lead) {
    fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) {
        if (CG == 1) tc::mbar_arrive(bar);
        else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(bar, lead)) : "memory");
    }
}

// How a mode's operands lie: the forward product's both along the contraction, ...
constexpr bool mn_major_a(int mode) { return mode == kGradWeight; }
constexpr bool mn_major_b(int mode) { return mode != kForward; }

template <int BN, int MODE, bool PROMOTE, int DT>
__global__ void __launch_bounds__(threads_of(epi_warps(PROMOTE && DT == GLR_F32)), 1) tc_product_kernel(const __grid_constant__ TcArgs a) {
    chain_begin();
    constexpr int CG = 2;
    constexpr bool MNA = mn_major_a(MODE), MNB = mn_major_b(MODE);
    constexpr bool PLANES = PROMOTE || MODE == kGradWeight;          // bf16 gradients of fp32 matrices too
    constexpr int kEpiWarps = epi_warps(PROMOTE && DT == GLR_F32), kCopyA = kEpiWarps, kCopyB = kEpiWarps + 1, kIssuer = kEpiWarps + 2, kSpan = BN / (kEpiWarps / 4);
    constexpr uint32_t SB = stage_bytes<BN, CG>();
    constexpr uint32_t kCols = 2 * BN;                               // two accumulators of BN columns
    extern __shared__ uint8_t dyn_smem[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
    float* blocks = reinterpret_cast<float*>(ring + static_cast<size_t>(a.stages) * SB);
    __shared__ __align__(8) uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = a.stages;
    const uint32_t rank = cluster_rank();
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    constexpr uint16_t both = 3;                      // the pair's CTAs
    volatile int* abort = &abort_flag;
    int* err = a.p.err;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int q = 0; q < S; ++q) { mbar_init(smem_u32(&full_bar[q]), 1); mbar_init(smem_u32(&empty_bar[q]), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&tfull_bar[b]), 1); mbar_init(smem_u32(&tempty_bar[b]), kEpiWarps * CG); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(kCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_base;

    if (warp == kCopyA || warp == kCopyB) {
        // one warp copies A, one B: an issue of copies takes a good hundred cycles, and a slab's products 512
        if (elect_one()) {
            const bool is_a = warp == kCopyA;
            int s = 0;
            uint32_t use = 0, issued = 0, last = 0;
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += step) {
                const Tile tl = tile_at<BN>(a, t);
                const int mine = tl.bn / CG;         // columns of the tile whose rows of B this CTA holds
                const int m0 = (tl.m * CG + static_cast<int>(rank)) * 128, n0 = tl.n0 + static_cast<int>(rank) * mine;
                for (int k = 0; k < a.slabs; ++k) {
                    if (!(ok = wait(smem_u32(&empty_bar[s]), use ^ 1u, abort, err))) break;
                    const uint32_t st = smem_u32(ring + static_cast<size_t>(s) * SB), bar = peer_addr(smem_u32(&full_bar[s]), 0);
                    if (is_a) {
                        if (rank == 0) mbar_expect_tx(smem_u32(&full_bar[s]), static_cast<uint32_t>(16384 + mine * 128) * CG);
                        load_a<CG, MNA, PLANES>(a, k, m0, tl.node, st, bar);
                    } else {
                        load_b<CG, MNB, PLANES>(a, k, n0, mine / 64, tl.node, st, bar);
                    }
                    issued |= 1u << s;
                    last = (last & ~(1u << s)) | (use << s);
                    if (++s == S) { s = 0; use ^= 1u; }
                }
            }
            if (!ok && rank == 0)                    // let the copies already issued land (both CTAs' arrive here)
                for (int q = 0; q < S; ++q)
                    if (issued & (1u << q))
                        for (int it = 0; it < 4000000 && !try_wait(smem_u32(&full_bar[q]), (last >> q) & 1u); ++it) __nanosleep(64);
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        if (rank == 0 && elect_one()) {
            int s = 0, b = 0;
            uint32_t use = 0, tuse[2] = {0, 0};
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += step) {
                const int bn = t < a.whole ? BN : BN / 2;
                for (int k0 = 0; k0 < a.slabs && ok; k0 += PROMOTE ? a.chunk : a.slabs) {
                    if (!(ok = wait(smem_u32(&tempty_bar[b]), tuse[b] ^ 1u, abort, err))) break;
                    fence_after();
                    const uint32_t d = tmem + static_cast<uint32_t>(b * BN);
                    const int k1 = PROMOTE ? min(k0 + a.chunk, a.slabs) : a.slabs;
                    for (int k = k0; k < k1; ++k) {
                        if (!(ok = wait(smem_u32(&full_bar[s]), use, abort, err))) break;
                        fence_after();
                        mma_stage<CG, MNA, MNB>(d, smem_u32(ring + static_cast<size_t>(s) * SB), bn, k > k0);
                        commit<CG>(smem_u32(&empty_bar[s]), both);
                        if (++s == S) { s = 0; use ^= 1u; }
                    }
                    if (!ok) break;
                    commit<CG>(smem_u32(&tfull_bar[b]), both);
                    tuse[b] ^= 1u;
                    b ^= 1;
                }
            }
        }
        __syncwarp();
    } else {
        // warp w: tensor-memory lanes 32 (w mod 4) .. + 31, the w / 4-th kSpan columns
        uint32_t tuse[2] = {0, 0};
        int b = 0;
        const int quad = warp & 3;
        float* block = blocks + warp * 32 * kBlockPitch;
        auto hand_back = [&]() { linear::hand_back<CG>(smem_u32(&tempty_bar[b]), 0); };
        for (int t = first; t < a.tiles; t += step) {
            const Tile tl = tile_at<BN>(a, t);
            const int span = tl.bn == BN ? kSpan : kSpan / 2, c0 = (warp >> 2) * span;
            if (PROMOTE) {
                // the chunks' sums are added up in registers, and put back into the last one's columns
                float sum[kSpan];
#pragma unroll
                for (int e = 0; e < kSpan; ++e) sum[e] = 0.f;
                bool ok = true;
                for (int k0 = 0; k0 < a.slabs; k0 += a.chunk) {
                    ok = wait(smem_u32(&tfull_bar[b]), tuse[b], abort, err);
                    if (!(ok = __all_sync(0xffffffffu, ok))) break;
                    fence_after();
                    const uint32_t ta = tmem + static_cast<uint32_t>(b * BN + c0) + (static_cast<uint32_t>(32 * quad) << 16);
#pragma unroll
                    for (int c = 0; c < kSpan; c += 16)
                        if (c < span) tmem_add16(ta + static_cast<uint32_t>(c), sum + c);
                    if (k0 + a.chunk < a.slabs) {
                        hand_back();
                        tuse[b] ^= 1u;
                        b ^= 1;
                    }
                }
                if (!ok) break;
                const uint32_t ta = tmem + static_cast<uint32_t>(b * BN + c0) + (static_cast<uint32_t>(32 * quad) << 16);
#pragma unroll
                for (int c = 0; c < kSpan; c += 32)
                    if (c < span) tmem_store32(ta + static_cast<uint32_t>(c), sum + c);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            } else {
                const bool ok = wait(smem_u32(&tfull_bar[b]), tuse[b], abort, err);
                if (!__all_sync(0xffffffffu, ok)) break;
                fence_after();
            }
            const int64_t i0 = static_cast<int64_t>(tl.m * CG + static_cast<int>(rank)) * 128 + 32 * quad;
            const uint32_t ta = tmem + static_cast<uint32_t>(b * BN + c0) + (static_cast<uint32_t>(32 * quad) << 16);
#pragma unroll 1
            for (int c = 0; c < span; c += 32) {
                const int64_t j = static_cast<int64_t>(tl.n0) + c0 + c + (lane & 3) * 8;
                // what the epilogue reads of the block, asked for before its sums are there
                constexpr bool AHEAD = !PROMOTE && MODE != kGradWeight;
                uint4 ahead[8];
                if (AHEAD && !a.columns) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int64_t i = i0 + 8 * q + (lane >> 2);
                        const bool in = i < a.p.M && j + 8 <= a.p.N;
                        if (in && a.p.add) ahead[q] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.p.add) + i * a.p.ldadd + j);
                        if (MODE == kGradInput && in && a.p.pre)
                            ahead[q + 4] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.p.pre) + i * a.p.ldpre + j);
                    }
                }
                float v[32];
                tmem_load32(ta + static_cast<uint32_t>(c), v);
                if (c + 32 >= span) hand_back();     // the last of this warp's columns
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 32; e += 4)
                    *reinterpret_cast<float4*>(block + lane * kBlockPitch + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                __syncwarp();
                if (a.columns) {
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        const int64_t j = static_cast<int64_t>(tl.n0) + c0 + c + lane;
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = block[(8 * q + e) * kBlockPitch + lane];
                        if (i0 + 8 * q < a.p.M && j < a.p.N) epilogue8<MODE, DT, true>(a, tl.node, i0 + 8 * q, j, w);
                    }
                    continue;
                }
#pragma unroll 1
                for (int q = 0; q < 4; ++q) {
                    const int r = 8 * q + (lane >> 2);
                    float w[8];
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        const float4 x = *reinterpret_cast<const float4*>(block + r * kBlockPitch + (lane & 3) * 8 + h);
                        w[h] = x.x; w[h + 1] = x.y; w[h + 2] = x.z; w[h + 3] = x.w;
                    }
                    if (i0 + r < a.p.M && j < a.p.N)
                        epilogue8<MODE, DT, false>(a, tl.node, i0 + r, j, w, AHEAD ? ahead : nullptr, AHEAD ? ahead + 4 : nullptr);
                    if (AHEAD) {                     // the loop is kept rolled: the next ones move up
#pragma unroll
                        for (int u = 0; u < 3; ++u) { ahead[u] = ahead[u + 1]; ahead[u + 4] = ahead[u + 5]; }
                    }
                }
            }
            tuse[b] ^= 1u;
            b ^= 1;
        }
    }
    fence_before();
    __syncthreads();
    cluster_sync();                                  // the cluster's barriers and tensor memory are done with
    if (warp == kIssuer) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
    }
}

// ------------------------------------------------------------------------------------------
// Few tiles: a cluster each, of CTAs with 128 x 64 of the result (CG = 1, two CTAs an SM) or of pairs with 256 x 256
// (CG = 2).  The cluster's q-th CTA or pair takes the q-th part of the stages, sums them in chunks, leaves its partial
// tile in shared memory (where the ring was) and finishes its part of the rows.
// ------------------------------------------------------------------------------------------
constexpr int kSplitN = 64;
template <int MODE, int CG>
__global__ void __launch_bounds__(threads_of(epi_warps(CG == 2)), CG == 2 ? 1 : 2) tc_split_kernel(const __grid_constant__ TcArgs a) {
    chain_begin();
    constexpr bool MNA = mn_major_a(MODE), MNB = mn_major_b(MODE);
    constexpr int BN = CG == 2 ? 256 : kSplitN, kPitch = BN + 4;
    constexpr int kEpiWarps = epi_warps(CG == 2), kCopyA = kEpiWarps, kCopyB = kEpiWarps + 1, kIssuer = kEpiWarps + 2;
    constexpr int kThreads = threads_of(kEpiWarps), kSpan = BN / (kEpiWarps / 4);
    constexpr uint32_t SB = stage_bytes<BN, CG>(), kCols = 2 * BN;
    extern __shared__ uint8_t dyn_smem[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = a.stages;
    const int splits = gridDim.y, split = blockIdx.y;
    const uint32_t half = CG == 2 ? cluster_rank() & 1 : 0, lead = CG == 2 ? cluster_rank() & ~1u : 0;    // of the pair
    const int k_first = static_cast<int>(static_cast<int64_t>(a.slabs) * split / splits);
    const int k_last = static_cast<int>(static_cast<int64_t>(a.slabs) * (split + 1) / splits);
    volatile int* abort = &abort_flag;
    int* err = a.p.err;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int q = 0; q < S; ++q) { mbar_init(smem_u32(&full_bar[q]), 1); mbar_init(smem_u32(&empty_bar[q]), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&tfull_bar[b]), 1); mbar_init(smem_u32(&tempty_bar[b]), kEpiWarps * CG); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) {
        if (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(kCols));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(kCols));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        }
    }
    fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_base;
    const Tile tl = tile_at<BN>(a, blockIdx.x / CG);
    const int m0 = (tl.m * CG + static_cast<int>(half)) * 128;
    float sum[kSpan];
#pragma unroll
    for (int e = 0; e < kSpan; ++e) sum[e] = 0.f;
    if (warp == kCopyA || warp == kCopyB) {
        if (elect_one()) {
            uint32_t issued = 0, last = 0;
            int s = 0;
            uint32_t use = 0;
            bool ok = true;
            for (int k = k_first; k < k_last; ++k) {
                if (!(ok = wait(smem_u32(&empty_bar[s]), use ^ 1u, abort, err))) break;
                const uint32_t own = smem_u32(&full_bar[s]), bar = CG == 2 ? peer_addr(own, lead) : own;
                const uint32_t st = smem_u32(ring + static_cast<size_t>(s) * SB);
                if (warp == kCopyA) {
                    if (half == 0) mbar_expect_tx(own, SB * CG);
                    load_a<CG, MNA, true>(a, k, m0, tl.node, st, bar);
                } else {
                    load_b<CG, MNB, true>(a, k, tl.n0 + static_cast<int>(half) * (BN / CG), BN / CG / 64, tl.node, st, bar);
                }
                issued |= 1u << s;
                last = (last & ~(1u << s)) | (use << s);
                if (++s == S) { s = 0; use ^= 1u; }
            }
            if (!ok && half == 0)                    // let the copies already issued land
                for (int q = 0; q < S; ++q)
                    if (issued & (1u << q))
                        for (int it = 0; it < 4000000 && !try_wait(smem_u32(&full_bar[q]), (last >> q) & 1u); ++it) __nanosleep(64);
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        if (half == 0 && elect_one()) {
            const uint16_t pair = static_cast<uint16_t>(3u << lead);
            int s = 0, b = 0;
            uint32_t use = 0, tuse[2] = {0, 0};
            bool ok = true;
            for (int k0 = k_first; k0 < k_last && ok; k0 += a.chunk) {
                if (!(ok = wait(smem_u32(&tempty_bar[b]), tuse[b] ^ 1u, abort, err))) break;
                fence_after();
                for (int k = k0; k < min(k0 + a.chunk, k_last); ++k) {
                    if (!(ok = wait(smem_u32(&full_bar[s]), use, abort, err))) break;
                    fence_after();
                    mma_stage<CG, MNA, MNB>(tmem + static_cast<uint32_t>(b * BN), smem_u32(ring + static_cast<size_t>(s) * SB), BN, k > k0);
                    commit<CG>(smem_u32(&empty_bar[s]), pair);
                    if (++s == S) { s = 0; use ^= 1u; }
                }
                if (!ok) break;
                commit<CG>(smem_u32(&tfull_bar[b]), pair);
                tuse[b] ^= 1u;
                b ^= 1;
            }
        }
        __syncwarp();
    } else {
        uint32_t tuse[2] = {0, 0};
        int b = 0;
        for (int k0 = k_first; k0 < k_last; k0 += a.chunk) {
            const bool ok = wait(smem_u32(&tfull_bar[b]), tuse[b], abort, err);
            if (!__all_sync(0xffffffffu, ok)) break;
            fence_after();
#pragma unroll
            for (int c = 0; c < kSpan; c += 16)
                tmem_add16(tmem + static_cast<uint32_t>(b * BN + (warp >> 2) * kSpan + c) + (static_cast<uint32_t>(32 * (warp & 3)) << 16), sum + c);
            hand_back<CG>(smem_u32(&tempty_bar[b]), lead);
            tuse[b] ^= 1u;
            b ^= 1;
        }
    }
    fence_before();
    __syncthreads();                                 // every stage has been read: the last products are done
    float* part = reinterpret_cast<float*>(ring);
    if (warp < kEpiWarps) {
        float* to = part + (32 * (warp & 3) + lane) * kPitch + (warp >> 2) * kSpan;
#pragma unroll
        for (int e = 0; e < kSpan; e += 4) *reinterpret_cast<float4*>(to + e) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
    }
    __syncthreads();
    if (CG == 2 || splits > 1) cluster_sync();
    const int rows = 128 / splits;                   // this CTA's rows of the tile, eight columns a thread
    for (int e = threadIdx.x; e < rows * (BN / 8); e += kThreads) {
        const int r = split * rows + (a.columns ? e / BN * 8 : e / (BN / 8)), c = a.columns ? e % BN : e % (BN / 8) * 8;
        const int64_t i = static_cast<int64_t>(m0) + r, j = static_cast<int64_t>(tl.n0) + c;
        if (i >= a.p.M || j >= a.p.N) continue;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = 0.f;
        for (int q = 0; q < splits; ++q) {
            const uint32_t from = peer_addr(smem_u32(part + r * kPitch + c), half + CG * q);
            if (a.columns) {
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    float x;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(from + 4 * kPitch * y) : "memory");
                    v[y] += x;
                }
                continue;
            }
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                float x[4];
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(from + 4 * h) : "memory");
#pragma unroll
                for (int y = 0; y < 4; ++y) v[h + y] += x[y];
            }
        }
        const bool wide32 = a.p.out_dtype == GLR_F32;
        if (a.columns) {
            if (wide32) epilogue8<MODE, GLR_F32, true>(a, tl.node, i, j, v);
            else epilogue8<MODE, GLR_BF16, true>(a, tl.node, i, j, v);
        } else {
            if (wide32) epilogue8<MODE, GLR_F32, false>(a, tl.node, i, j, v);
            else epilogue8<MODE, GLR_BF16, false>(a, tl.node, i, j, v);
        }
    }
    if (CG == 2 || splits > 1) cluster_sync();       // the peers are done with this CTA's shared memory
    else __syncthreads();
    if (warp == kIssuer) {
        fence_after();
        if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
    }
}

// Rows of `cols` elements, ld apart, as `planes` bf16 matrices in rows of ldp (a multiple of eight), one after the
// other: x = hi + mid + lo, each the bf16 nearest to what is left; an infinity is 1, 0 and itself, so that it meets the
// other operand's first plane alone (times a lower one of 0, or of the other sign, an infinity would be NaN).  One or
// two matrices a launch, eight neighbouring elements a thread, 2 to 256 threads (a power of two) a row.  Bound by HBM.
constexpr int kPackThreads = 256;
struct PackJob {
    const void* x; int64_t rows, cols, ld;
    __nv_bfloat16* to; int64_t ldp;
    int shift;                                       // log2 of the threads a row
    int wide;                                        // 16-byte loads
};
struct PackArgs { PackJob job[2]; int planes; };
template <class T>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const __grid_constant__ PackArgs a) {
    chain_begin();
    __shared__ __align__(16) T turn[kPackThreads * 8];
    const PackJob& x = a.job[blockIdx.y];
    const int per = 1 << x.shift, lane = threadIdx.x & 31;
    T* mine = turn + (threadIdx.x & ~31) * 8;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (kPackThreads >> x.shift);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kPackThreads >> x.shift) + (threadIdx.x >> x.shift); i < x.rows; i += step) {
        const T* row = static_cast<const T*>(x.x) + i * x.ld;
        for (int64_t j = (threadIdx.x & (per - 1)) * 8; j < x.ldp; j += per * 8) {
            const int n = static_cast<int>(min(static_cast<int64_t>(8), x.cols - j));
            float v[8];
            const int64_t first = j - lane * 8;
            if (!x.wide && per >= 32 && first + 256 <= x.ldp) {
                // a warp's 256 elements of a row, neighbouring lanes' next to each other, turned round in shared memory
#pragma unroll
                for (int e = 0; e < 8; ++e) mine[e * 32 + lane] = first + e * 32 + lane < x.cols ? row[first + e * 32 + lane] : T(0.f);
                __syncwarp();
                get8(mine, lane * 8, 8, true, sizeof(T) == 2 ? GLR_BF16 : GLR_F32, v);
                __syncwarp();
            } else {
                get8(row, j, n, x.wide, sizeof(T) == 2 ? GLR_BF16 : GLR_F32, v);
            }
            constexpr float kMost = 3.3895313892515355e38f;      // bf16's largest
            float most = 0.f;                        // (a NaN needs no care)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
            const bool careful = most > kMost;
            for (int p = 0; p < a.planes; ++p) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * q], v[2 * q + 1]);
                    if (careful) {
                        auto plane = [&](float x, __nv_bfloat16& to) {
                            if (isinf(x)) {
                                if (a.planes == 3 && p < 2) to = __float2bfloat16_rn(p == 0 ? copysignf(1.f, x) : 0.f);
                            } else if (isinf(__bfloat162float(to))) {
                                to = __float2bfloat16_rz(x);     // what would round up to infinity is cut off
                            }
                        };
                        plane(v[2 * q], h.x);
                        plane(v[2 * q + 1], h.y);
                    }
                    w[q] = *reinterpret_cast<const uint32_t*>(&h);
                    if (!careful || !isinf(v[2 * q])) v[2 * q] -= __low2float(h);
                    if (!careful || !isinf(v[2 * q + 1])) v[2 * q + 1] -= __high2float(h);
                }
                *reinterpret_cast<uint4*>(x.to + (p * x.rows + i) * x.ldp + j) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

bool on16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// An operand as its storage: `rows` rows of `cols` contiguous elements ld apart (all nodes' rows together).
struct Storage { int64_t rows, cols, ld; };
Storage storage(int64_t si, int64_t sp, int64_t ni, int64_t np, int nodes) {
    return sp == 1 ? Storage{ni, np, si} : Storage{np * nodes, ni, sp};
}
int64_t up8(int64_t x) { return (x + 7) / 8 * 8; }

// The tile copies of an operand X(i, p): rows of 64 contraction elements (K-major), or 64 x 64 blocks of
// (index, contraction) per node (MN-major); planes one after the other.
bool operand_map(CUtensorMap* map, const void* x, int64_t si, int64_t sp, int64_t sb, int64_t ni, int64_t np, int nodes, int planes,
                 uint32_t rows) {
    // a stride along a single row or plane is never used; the copies only want it to be valid
    if (ni == 1 && sp == 1) si = up8(np);
    if (np == 1 && sp != 1) sp = up8(ni);
    if (sp == 1) {
        const uint64_t dims[3] = {static_cast<uint64_t>(np), static_cast<uint64_t>(ni), static_cast<uint64_t>(planes)};
        const uint64_t str[2] = {static_cast<uint64_t>(si) * 2, static_cast<uint64_t>(si * ni) * 2};
        const uint32_t box[3] = {kSlab, rows, 1};
        return host::encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, 3, dims, str, box, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    const uint64_t dims[3] = {static_cast<uint64_t>(ni), static_cast<uint64_t>(np), static_cast<uint64_t>(nodes * planes)};
    const uint64_t str[2] = {static_cast<uint64_t>(sp) * 2, static_cast<uint64_t>(nodes * planes > 1 ? sb : sp) * 2};
    const uint32_t box[3] = {64, kSlab, 1};
    return host::encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, 3, dims, str, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <class Kernel>
cudaError_t launch(Kernel kernel, const TcArgs& a, dim3 grid, dim3 cluster, int threads, size_t smem, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster.x; attr[1].val.clusterDim.y = cluster.y; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = threads; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}
template <int MODE>
cudaError_t launch_mode(TcArgs& a, bool promote, int splits, bool paired, int sms, cudaStream_t st) {
    if (splits && !paired) {
        // half of an SM's shared memory: two CTAs an SM
        a.stages = 4;
        const size_t smem = a.stages * stage_bytes<kSplitN, 1>() + 1024;
        return launch(tc_split_kernel<MODE, 1>, a, dim3(static_cast<unsigned>(a.tiles), splits), dim3(1, splits), threads_of(epi_warps(false)), smem, st);
    }
    if (splits) {
        a.stages = 6;
        const size_t smem = a.stages * stage_bytes<256, 2>() + 1024;
        return launch(tc_split_kernel<MODE, 2>, a, dim3(static_cast<unsigned>(2 * a.tiles), splits), dim3(2, splits), threads_of(epi_warps(true)), smem, st);
    }
    const uint32_t sb = stage_bytes<256, 2>();
    const int epi = epi_warps(a.p.out_dtype == GLR_F32);
    const size_t blocks = epi * kBlockBytes;
    a.stages = std::min<int>(kMaxStages, static_cast<int>((kSmemBytes - 1024 - blocks) / sb));
    const size_t smem = static_cast<size_t>(a.stages) * sb + 1024 + blocks;
    const dim3 grid(static_cast<unsigned>(std::min(a.tiles, sms / 2) * 2));
    if (promote && a.p.out_dtype == GLR_BF16)
        return launch(tc_product_kernel<256, MODE, true, GLR_BF16>, a, grid, dim3(2), threads_of(epi), smem, st);
    return promote ? launch(tc_product_kernel<256, MODE, true, GLR_F32>, a, grid, dim3(2), threads_of(epi), smem, st)
                   : launch(tc_product_kernel<256, MODE, false, GLR_BF16>, a, grid, dim3(2), threads_of(epi), smem, st);
}

// A matrix to pack: its threads a row.
PackJob pack_job(const void* x, const Storage& s, int64_t esize, void* to) {
    PackJob j{x, s.rows, s.cols, s.ld, static_cast<__nv_bfloat16*>(to), up8(s.cols), 1, on16(x) && s.ld * esize % 16 == 0};
    while (j.shift < 8 && (8 << j.shift) < j.ldp) ++j.shift;
    return j;
}
template <class T>
cudaError_t pack(const PackArgs& a, int jobs, cudaStream_t st) {
    int64_t blocks = 1;
    for (int q = 0; q < jobs; ++q) blocks = std::max(blocks, (a.job[q].rows + (kPackThreads >> a.job[q].shift) - 1) / (kPackThreads >> a.job[q].shift));
    return launch_chain(pack_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>(blocks, 152 * 16)), jobs), kPackThreads, 0, st, a);
}

int64_t big_tiles(const Product& p) { return ((p.M + 255) / 256) * ((p.N + 255) / 256) * p.nodes; }
int64_t small_tiles(const Product& p) { return ((p.M + 127) / 128) * ((p.N + kSplitN - 1) / kSplitN) * p.nodes; }
// One of three, by the cycles it takes (measured; a stage is a slab, or one of an fp32 slab's six products).
// 256 x 256 tiles, one after the other on every pair: 530 a stage, 650 with promoted sums.  The same tiles, two
// pairs sharing a contraction: 670 a stage, and more to begin and end with; 36 such clusters run at once on 152 SMs
// (four pairs to a tile: too few clusters at once, never the fastest).  128 x 64 tiles shared by one to eight CTAs: 420 a
// stage, 620 with two on an SM.  400 x 4096 x 4096 fp32: 176, 114 and 157 us; 1000 x 11008 x 2048 bf16: 56, 48 and 66; 200 x
// 4096 x 4096 bf16: 27, 27 and 23; 24 rows: 27, 25 and 19.
// Contractions up to which the sums of whole tiles for bf16 results are truncated throughout: of positive matrices, 32768 rows'
// gradients come out 2^-12.5 of their value short (fp32 ones 2^-12.0), a sixteenth of the rounding to bf16, 2^20 rows' 2^-7.3.
// Beyond it they are promoted too (2^-16), in chunks of sixteen times the length, whose reads of tensor memory do not show, by
// eight warps: with sixteen a stage of the ring less (8192 x 4096 over 131072: 4.8 to 5.0 ms, truncated 4.9; with sixteen 5.4).
constexpr int64_t kMostTruncated = 32768;
constexpr int kLongChunk = 16;
struct Choice { int splits; bool paired; int64_t cycles; };
Choice choose(const Product& p, int64_t slabs, bool promote, int sms) {
    const int64_t big = big_tiles(p), small = small_tiles(p), pairs = sms / 2;
    const auto waves = [](int64_t n, int64_t at_once) { return (n + at_once - 1) / at_once; };
    int64_t best = 4000 + waves(big, pairs) * slabs * (promote ? 650 : 530);
    int splits = 0;
    bool paired = false;
    if (const int64_t t = 26000 + waves(big, sms * 36 / 152) * (slabs + 1) / 2 * 670; t < best && slabs >= 8) { best = t; splits = 2; paired = true; }
    for (int q = 1; q <= 8 && (q == 1 || slabs >= 4 * q); q *= 2) {
        const int64_t t = 2000 + waves(small * q, 2 * sms) * (6000 + waves(slabs, q) * (small * q > sms ? 620 : 420));
        if (t < best) { best = t; splits = q; paired = false; }
    }
    return {splits, paired, best};
}

// Whether an operand's rows lie on 16 bytes as they are.
bool lies_well(const void* x, int64_t si, int64_t sp, int64_t sb, int64_t ni, int64_t np, int nodes) {
    const int64_t ld = sp == 1 ? si : sp, rows = sp == 1 ? ni : np;
    return on16(x) && (rows == 1 || (ld % 8 == 0 && ld < (int64_t(1) << 36))) && (nodes == 1 || (sb % 8 == 0 && sb < (int64_t(1) << 36)));
}

}  // namespace

int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) return sms;
    cudaGetLastError();
    return 152;
}

// Which operands a product has to have packed, and what that takes.
TcPlan tc_plan(const Product& p) {
    TcPlan t{};
    if (p.K <= 0 || p.M <= 0 || p.N <= 0) return t;
    // (single columns may lie along the contraction in a mode that has them across it)
    if ((p.sAp != 1) != mn_major_a(p.mode) || (p.sBp != 1) != mn_major_b(p.mode)) return t;
    t.planes = p.dtype == GLR_F32 ? 3 : 1;
    t.pack_a = t.planes == 3 || !lies_well(p.A, p.sAi, p.sAp, p.sAb, p.M, p.K, p.nodes);
    t.pack_b = t.planes == 3 || !lies_well(p.B, p.sBj, p.sBp, p.sBb, p.N, p.K, p.nodes);
    const Storage a = storage(p.sAi, p.sAp, p.M, p.K, p.nodes), b = storage(p.sBj, p.sBp, p.N, p.K, p.nodes);
    if (t.pack_a) t.bytes_a = (t.planes * a.rows * up8(a.cols) * 2 + 255) / 256 * 256;
    if (t.pack_b) t.bytes_b = t.planes * b.rows * up8(b.cols) * 2;
    if (!t.pack_a && !t.pack_b) {
        t.ok = true;
        return t;
    }
    // Packing reads and writes the matrices once more, in a launch of its own (2 us for a million fp32 elements, 0.9 for
    // bf16); any_product does without.  Both times are estimated.  Rows off 16 bytes, bf16: 3 x 4096 x 4096 81 us unpacked,
    // 48 packed, 128 x 1500 x 1500 38 and 19, 64 x 500 x 500 13 and 17; fp32: 16 x 4096 x 4096 91 and 74, 300 x 1500 x
    // 1500 58 and 33, 32 x 8000 x 1000 44 and 52; fewer fp32 rows stay unpacked (three of 4096 x 4096 89 and 142: the few
    // lines of their planes are read by all SMs at once).
    const double flops = 2.0 * static_cast<double>(p.M) * static_cast<double>(p.N) * static_cast<double>(p.K) * p.nodes;
    if (flops < 1e7 || (t.planes == 3 && p.M < 16)) return t;
    const int64_t slabs = (p.K + kSlab - 1) / kSlab * (t.planes == 3 ? 6 : 1);
    const double elements = (t.pack_a ? static_cast<double>(a.rows) * a.cols : 0.0) + (t.pack_b ? static_cast<double>(b.rows) * b.cols : 0.0);
    const double packed = (t.planes == 3 ? 13 + 2e-6 * elements : 11 + 9e-7 * elements) + choose(p, slabs, p.out_dtype == GLR_F32, sm_count()).cycles / 1870.0;
    t.ok = packed < any_cost(p);
    return t;
}

cudaError_t tc_product(const Product& p, const TcPlan& plan, void* workspace, cudaStream_t st) {
    TcArgs a{};
    a.p = p;
    Product& q = a.p;
    cudaError_t e = cudaSuccess;
    PackArgs jobs{};
    jobs.planes = plan.planes;
    int n = 0;
    auto packed = [&](const void*& x, int64_t& si, int64_t& sp, int64_t& sb, int64_t ni, uint8_t* to) {
        const Storage s = storage(si, sp, ni, p.K, p.nodes);
        jobs.job[n++] = pack_job(x, s, plan.planes == 3 ? 4 : 2, to);
        x = to;
        (sp == 1 ? si : sp) = up8(s.cols);
        sb = sp == 1 ? 0 : p.K * sp;
    };
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (plan.pack_a) packed(q.A, q.sAi, q.sAp, q.sAb, p.M, ws);
    if (plan.pack_b) packed(q.B, q.sBj, q.sBp, q.sBb, p.N, ws + plan.bytes_a);
    if (n && (e = plan.planes == 3 ? pack<float>(jobs, n, st) : pack<__nv_bfloat16>(jobs, n, st)) != cudaSuccess) return e;
    const int sms = sm_count();
    const bool fp32 = p.out_dtype == GLR_F32, promote = fp32 || p.K > kMostTruncated;
    a.planes = plan.planes;
    a.chunk = plan.planes == 3 ? 6 : 4;
    const int64_t slabs = (p.K + kSlab - 1) / kSlab * (plan.planes == 3 ? 6 : 1);
    if (slabs > (1 << 30)) return cudaErrorInvalidValue;
    a.slabs = static_cast<int>(slabs);
    const Choice how = choose(p, slabs, fp32, sms);
    if (!fp32 && !how.splits) a.chunk *= kLongChunk;
    const int64_t big = big_tiles(p), small = small_tiles(p), pairs = sms / 2;
    if (std::max(big, small) > (1 << 30)) return cudaErrorInvalidValue;
    const int splits = how.splits;
    const bool paired = how.paired;
    const int bm = splits && !paired ? 128 : 256, bn = splits && !paired ? kSplitN : 256;
    a.tiles_m = static_cast<int>((p.M + bm - 1) / bm);
    a.tiles_n = static_cast<int>((p.N + bn - 1) / bn);
    a.tiles = a.whole = static_cast<int>(splits && !paired ? small : big);
    if (!splits) {
        // a last wave of at most half the pairs: half tiles, one for each of twice as many
        const int rest = static_cast<int>(big % pairs);
        if (rest > 0 && 2 * rest <= pairs) { a.whole -= rest; a.tiles += rest; }
    }
    const int64_t os = p.out_dtype == GLR_BF16 ? 2 : 4, per16 = 16 / os;
    if (p.mode == kGradWeight) {
        a.wide = p.N * os % 16 == 0;
        for (int i = 0; i < p.nodes; ++i) a.wide = a.wide && on16(p.outs[i]);
    } else {
        a.wide = (on16(p.out) && p.ldo % per16 == 0 ? 1 : 0) | (on16(p.bias) ? 2 : 0) | (on16(p.add) && p.ldadd % per16 == 0 ? 4 : 0) |
                 (on16(p.pre) && p.ldpre % per16 == 0 ? 8 : 0) | (on16(p.aux) && p.ldaux % per16 == 0 ? 16 : 0);
    }
    const int need = p.mode == kGradWeight ? 1 : 1 | (p.add ? 4 : 0) | (p.pre ? 8 : 0) | (p.aux ? 16 : 0);
    a.columns = (a.wide & need) != need;
    if (!operand_map(&a.mapA, q.A, q.sAi, q.sAp, q.sAb, p.M, p.K, p.nodes, a.planes, 128) ||
        !operand_map(&a.mapB, q.B, q.sBj, q.sBp, q.sBb, p.N, p.K, p.nodes, a.planes, 64))
        return cudaErrorInvalidValue;
    return p.mode == kForward ? launch_mode<kForward>(a, promote, splits, paired, sms, st)
         : p.mode == kGradInput ? launch_mode<kGradInput>(a, promote, splits, paired, sms, st)
                                : launch_mode<kGradWeight>(a, promote, splits, paired, sms, st);
}

}  // namespace linear
}  // namespace glr
