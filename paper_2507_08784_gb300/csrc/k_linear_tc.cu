// Products of linear layers on the fifth-generation tensor cores: out = epilogue(A B^T) for bf16 operands
// whose rows lie on 16 bytes, either operand contiguous along the contraction ("K-major") or along its own
// index ("MN-major"), so that the forward product, the input's gradient and the weights' gradients all read
// their matrices as they are.
//
// One persistent kernel: a CTA (CG = 1) or a pair of CTAs on two SMs (CG = 2) takes 128 CG x BN output
// tiles in turn.  One warp copies operand slabs of 64 contraction elements (128-byte swizzle) into a ring of
// shared-memory stages, one thread issues tcgen05.mma.kind::f16 (of the pair's first CTA: each CTA holds its
// 128 rows of A and half of B's, and the result's rows stay in their CTA's tensor memory), and eight warps
// bring the finished accumulator through the epilogue while the next tile's products run into the other half
// of tensor memory.  Stages are handed over on mbarriers; every wait is bounded: a CTA that gives up counts
// the event, lets its copies land, frees tensor memory and returns.
//
// What bounds it: the tensor pipe for contractions of about 1000 and more; below that the epilogue, which
// each thread does on a row of the tile, 16 bytes a load or store.
#include <algorithm>

#include "glr_host.cuh"
#include "glr_linear.cuh"
#include "glr_ptx.cuh"

namespace glr {
namespace linear {

namespace {

using tc::fence_after;
using tc::fence_before;
using tc::mbar_expect_tx;
using tc::mbar_init;
using tc::smem_u32;

constexpr int kEpiWarps = 8, kProducer = 8, kIssuer = 9, kThreads = 320;
constexpr int kSlab = 64;                       // contraction elements a stage: one 128-byte swizzle row of bf16
constexpr int kMaxStages = 8;
constexpr size_t kRingBytes = 208 * 1024;
constexpr int kBand = 8;                        // tile rows walked together, so that a wave's operands share L2

struct TcArgs {
    Product p;
    CUtensorMap mapA, mapB;
    int tiles_m, tiles_n, tiles, slabs, stages;
    int wide;                                   // 16-byte accesses: bit 0 out, 1 bias, 2 add, 3 pre, 4 aux
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
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
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
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
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
// Arrives on `bar` (of both CTAs of a pair) when the products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
    if (CG == 1) tc::mma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
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

// Eight bf16 at p (n of them in range), widened.
__device__ __forceinline__ void get8(const void* base, int64_t at, int n, bool wide, float (&v)[8]) {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + at;
    if (wide && n == 8) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[2 * q] = __uint_as_float(w[q] << 16);
            v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? __bfloat162float(p[e]) : 0.f;
    }
}
__device__ __forceinline__ void put8(void* base, int64_t at, int n, bool wide, int dtype, const float (&v)[8]) {
    if (dtype == GLR_F32) {
        float* p = static_cast<float*>(base) + at;
        if (wide && n == 8) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (e < n) p[e] = v[e];
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
        for (int e = 0; e < 8; ++e) if (e < n) p[e] = __float2bfloat16_rn(v[e]);
    }
}
template <bool SLOPE>
__device__ __forceinline__ void act8(float (&v)[8], int act) {
    switch (act) {                               // one branch for the eight
#define GLR_ACT_CASE(A)                                                                               \
        case A:                                                                                       \
            _Pragma("unroll") for (int e = 0; e < 8; ++e) v[e] = SLOPE ? act_slope(v[e], A) : act_value(v[e], A); \
            break;
        GLR_ACT_CASE(GLR_ACT_RELU)
        GLR_ACT_CASE(GLR_ACT_GELU)
        GLR_ACT_CASE(GLR_ACT_GELU_TANH)
        GLR_ACT_CASE(GLR_ACT_SILU)
#undef GLR_ACT_CASE
        default: break;
    }
}

// The epilogue on eight neighbouring columns of a row (i, j): acc in v.
__device__ __forceinline__ void epilogue8(const TcArgs& a, int node, int64_t i, int64_t j, float (&v)[8]) {
    const Product& p = a.p;
    const int n = static_cast<int>(p.N - j < 8 ? p.N - j : 8);
    if (p.mode == kGradWeight) {
        put8(p.outs[node], i * p.N + j, n, a.wide & 1, p.out_dtype, v);
        return;
    }
    float x[8];
    if (p.mode == kForward) {
        if (p.bias) {
            get8(p.bias, j, n, a.wide & 2, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += x[e];
        }
        if (p.aux) put8(p.aux, i * p.ldaux + j, n, a.wide & 16, GLR_BF16, v);
        act8<false>(v, p.act);
        if (p.add) {
            get8(p.add, i * p.ldadd + j, n, a.wide & 4, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += x[e];
        }
    } else {
        if (p.add) {
            get8(p.add, i * p.ldadd + j, n, a.wide & 4, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += x[e];
        }
        if (p.aux) put8(p.aux, i * p.ldaux + j, n, a.wide & 16, GLR_BF16, v);
        if (p.pre) {
            get8(p.pre, i * p.ldpre + j, n, a.wide & 8, x);
            act8<true>(x, p.act);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= x[e];
        }
    }
    put8(p.out, i * p.ldo + j, n, a.wide & 1, GLR_BF16, v);
}

struct Tile { int node, m, n; };
__device__ __forceinline__ Tile tile_at(const TcArgs& a, int t) {
    const int per = a.tiles_m * a.tiles_n;
    Tile r;
    r.node = t / per;
    t -= r.node * per;
    const int band = t / (kBand * a.tiles_n), in = t - band * kBand * a.tiles_n;
    const int h = min(kBand, a.tiles_m - band * kBand);
    r.m = band * kBand + in % h;
    r.n = in / h;
    return r;
}

template <int BN, int CG, bool MNA, bool MNB>
__global__ void __launch_bounds__(kThreads, 1) tc_product_kernel(const __grid_constant__ TcArgs a) {
    chain_begin();
    constexpr uint32_t SB = stage_bytes<BN, CG>(), BB = BN / CG;     // bytes a stage, rows of B in this CTA
    constexpr uint32_t kCols = 2 * BN;                               // two accumulators of BN columns
    extern __shared__ uint8_t dyn_smem[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = a.stages;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
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

    if (warp == kProducer) {
        if (lane == 0) {
            int s = 0;
            uint32_t use = 0, issued = 0, last = 0;
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += step) {
                const Tile tl = tile_at(a, t);
                const int m0 = (tl.m * CG + static_cast<int>(rank)) * 128, n0 = tl.n * BN + static_cast<int>(rank) * static_cast<int>(BB);
                for (int k = 0; k < a.slabs; ++k) {
                    if (!(ok = wait(smem_u32(&empty_bar[s]), use ^ 1u, abort, err))) break;
                    const uint32_t st = smem_u32(ring + static_cast<size_t>(s) * SB);
                    uint32_t bar = smem_u32(&full_bar[s]);
                    if (rank == 0) mbar_expect_tx(bar, SB * CG);
                    else bar = peer_addr(bar, 0);
                    if (MNA) {
                        for (int c = 0; c < 2; ++c) load_3d<CG>(st + c * 8192, &a.mapA, m0 + 64 * c, k * kSlab, tl.node, bar);
                    } else {
                        load_2d<CG>(st, &a.mapA, k * kSlab, m0, bar);
                    }
                    if (MNB) {
                        for (int c = 0; c < static_cast<int>(BB) / 64; ++c)
                            load_3d<CG>(st + 16384 + c * 8192, &a.mapB, n0 + 64 * c, k * kSlab, tl.node, bar);
                    } else {
                        load_2d<CG>(st + 16384, &a.mapB, k * kSlab, n0, bar);
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
        if (lane == 0 && rank == 0) {
            constexpr uint32_t id = (1u << 4) | (1u << 7) | (1u << 10) | (MNA ? 1u << 15 : 0u) | (MNB ? 1u << 16 : 0u) |
                                    (static_cast<uint32_t>(BN >> 3) << 17) | (static_cast<uint32_t>(8 * CG) << 24);
            int s = 0, b = 0;
            uint32_t use = 0, tuse[2] = {0, 0};
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += step) {
                if (!(ok = wait(smem_u32(&tempty_bar[b]), tuse[b] ^ 1u, abort, err))) break;
                fence_after();
                const uint32_t d = tmem + static_cast<uint32_t>(b * BN);
                for (int k = 0; k < a.slabs; ++k) {
                    if (!(ok = wait(smem_u32(&full_bar[s]), use, abort, err))) break;
                    fence_after();
                    const uint32_t st = smem_u32(ring + static_cast<size_t>(s) * SB);
#pragma unroll
                    for (int kk = 0; kk < kSlab / 16; ++kk)
                        mma_f16<CG>(d, operand_desc(st + (MNA ? 2048 : 32) * kk, MNA, 8192),
                                    operand_desc(st + 16384 + (MNB ? 2048 : 32) * kk, MNB, 8192), id, (k | kk) ? 1u : 0u);
                    commit<CG>(smem_u32(&empty_bar[s]));
                    if (++s == S) { s = 0; use ^= 1u; }
                }
                if (!ok) break;
                commit<CG>(smem_u32(&tfull_bar[b]));
                tuse[b] ^= 1u;
                b ^= 1;
            }
        }
        __syncwarp();
    } else {
        // warp w: tensor-memory lanes 32 (w mod 4) .. + 31, columns of half w / 4
        uint32_t tuse[2] = {0, 0};
        int b = 0;
        const int quad = warp & 3, c0 = (warp >> 2) * (BN / 2);
        for (int t = first; t < a.tiles; t += step) {
            const Tile tl = tile_at(a, t);
            const bool ok = wait(smem_u32(&tfull_bar[b]), tuse[b], abort, err);
            if (!__all_sync(0xffffffffu, ok)) break;
            fence_after();
            const int64_t i = static_cast<int64_t>(tl.m * CG + static_cast<int>(rank)) * 128 + 32 * quad + lane;
            const uint32_t ta = tmem + static_cast<uint32_t>(b * BN + c0) + (static_cast<uint32_t>(32 * quad) << 16);
#pragma unroll 1
            for (int c = 0; c < BN / 2; c += 32) {
                float v[32];
                tmem_load32(ta + static_cast<uint32_t>(c), v);
                if (c + 32 >= BN / 2) {              // the last of this warp's columns: hand the accumulator back
                    fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        const uint32_t bar = smem_u32(&tempty_bar[b]);
                        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(CG == 1 ? peer_addr(bar, cluster_rank()) : peer_addr(bar, 0)) : "memory");
                    }
                }
                const int64_t j = static_cast<int64_t>(tl.n) * BN + c0 + c;
                if (i < a.p.M) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = v[8 * q + e];
                        if (j + 8 * q < a.p.N) epilogue8(a, tl.node, i, j + 8 * q, w);
                    }
                }
            }
            tuse[b] ^= 1u;
            b ^= 1;
        }
    }
    fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();                     // the pair's barriers and tensor memory are done with
    if (warp == kIssuer) {
        fence_after();
        if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
    }
}

bool on16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The tile copies of an operand X(i, p): rows of 64 contraction elements (K-major), or 64 x 64 blocks of
// (index, contraction) per node (MN-major).
bool operand_map(CUtensorMap* map, const void* x, int64_t si, int64_t sp, int64_t sb, int64_t ni, int64_t np, int nodes, uint32_t rows) {
    // a stride along a single row is never used; the copies only want it to be valid
    if (ni == 1 && sp == 1) si = (np + 7) / 8 * 8;
    if (np == 1 && sp != 1) sp = (ni + 7) / 8 * 8;
    if (sp == 1) {
        const uint64_t dims[2] = {static_cast<uint64_t>(np), static_cast<uint64_t>(ni)}, str[1] = {static_cast<uint64_t>(si) * 2};
        const uint32_t box[2] = {kSlab, rows};
        return host::encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, 2, dims, str, box, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    const uint64_t dims[3] = {static_cast<uint64_t>(ni), static_cast<uint64_t>(np), static_cast<uint64_t>(nodes)};
    const uint64_t str[2] = {static_cast<uint64_t>(sp) * 2, static_cast<uint64_t>(nodes > 1 ? sb : sp) * 2};
    const uint32_t box[3] = {64, kSlab, 1};
    return host::encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, 3, dims, str, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int BN, int CG, bool MNA, bool MNB>
cudaError_t launch(TcArgs& a, cudaStream_t st) {
    constexpr uint32_t SB = stage_bytes<BN, CG>();
    a.stages = std::min<int>(kMaxStages, static_cast<int>(kRingBytes / SB));
    const size_t smem = std::max<size_t>(static_cast<size_t>(a.stages) * SB + 1024, 120 * 1024);
    auto kernel = tc_product_kernel<BN, CG, MNA, MNB>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    int dev = 0, sms = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = static_cast<unsigned>(std::min(a.tiles, sms / CG) * CG);
    cfg.blockDim = kThreads; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}
template <int BN, int CG>
cudaError_t launch_major(TcArgs& a, bool mna, bool mnb, cudaStream_t st) {
    if (mna) return mnb ? launch<BN, CG, true, true>(a, st) : launch<BN, CG, true, false>(a, st);
    return mnb ? launch<BN, CG, false, true>(a, st) : launch<BN, CG, false, false>(a, st);
}

}  // namespace

bool tc_ok(const Product& p) {
    auto operand = [&](const void* x, int64_t si, int64_t sp, int64_t sb, int64_t ni) {
        const int64_t ld = sp == 1 ? si : sp, rows = sp == 1 ? ni : p.K;
        return on16(x) && (rows == 1 || (ld % 8 == 0 && ld < (int64_t(1) << 36))) &&
               (p.nodes == 1 || (sb % 8 == 0 && sb < (int64_t(1) << 36)));
    };
    return p.dtype == GLR_BF16 && p.K > 0 && p.M > 0 && p.N > 0 && operand(p.A, p.sAi, p.sAp, p.sAb, p.M) &&
           operand(p.B, p.sBj, p.sBp, p.sBb, p.N);
}

cudaError_t tc_product(const Product& p, cudaStream_t st) {
    TcArgs a{};
    a.p = p;
    const bool mna = p.sAp != 1, mnb = p.sBp != 1;
    const int BN = 256, CG = 2;
    a.tiles_m = static_cast<int>((p.M + 128 * CG - 1) / (128 * CG));
    a.tiles_n = static_cast<int>((p.N + BN - 1) / BN);
    const int64_t tiles = static_cast<int64_t>(a.tiles_m) * a.tiles_n * p.nodes;
    if (tiles > (1 << 30)) return cudaErrorInvalidValue;
    a.tiles = static_cast<int>(tiles);
    a.slabs = static_cast<int>((p.K + kSlab - 1) / kSlab);
    const int64_t os = p.out_dtype == GLR_BF16 ? 2 : 4;
    if (p.mode == kGradWeight) {
        a.wide = p.N * os % 16 == 0;
        for (int i = 0; i < p.nodes; ++i) a.wide = a.wide && on16(p.outs[i]);
    } else {
        a.wide = (on16(p.out) && p.ldo % 8 == 0 ? 1 : 0) | (on16(p.bias) ? 2 : 0) | (on16(p.add) && p.ldadd % 8 == 0 ? 4 : 0) |
                 (on16(p.pre) && p.ldpre % 8 == 0 ? 8 : 0) | (on16(p.aux) && p.ldaux % 8 == 0 ? 16 : 0);
    }
    if (!operand_map(&a.mapA, p.A, p.sAi, p.sAp, p.sAb, p.M, p.K, p.nodes, 128) ||
        !operand_map(&a.mapB, p.B, p.sBj, p.sBp, p.sBb, p.N, p.K, p.nodes, BN / CG))
        return cudaErrorInvalidValue;
    return launch_major<256, 2>(a, mna, mnb, st);
}

}  // namespace linear
}  // namespace glr
