// Products of linear layers with their epilogues, for any sizes, strides and alignment: 64 x 64 output
// tiles by four warps, operand slabs of 32 contraction elements through registers (two slabs ahead) into shared
// memory.  Where the tiles leave SMs idle a cluster of up to eight CTAs shares a tile's contraction; their partial
// tiles are added over distributed shared memory in the order of the contraction, each CTA finishing its rows.
// It takes what is too small to be laid out for the tensor cores' own kernels, and calls without workspace.
// Bound by the loads' latency in the chain of slabs at these sizes (300 x 500 x 500 fp32: 19 us with its launch).
// bf16 operands go through mma.sync.m16n8k16; fp32 ones through m16n8k8 in the 3xTF32 form
// (x = hi + lo, a b ~ hi hi + hi lo + lo hi, a few 2^-21 relative a product), accumulated in fp32.
#include "glr_linear.cuh"

namespace glr {
namespace linear {

namespace {

constexpr int kTile = 64, kSlab = 32, kThreads = 128;

template <class T> struct Traits;
template <> struct Traits<float> { static constexpr int kVec = 4, kPitch = 36; };
template <> struct Traits<__nv_bfloat16> { static constexpr int kVec = 8, kPitch = 40; };

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float get(const void* p, int64_t i, int dtype) {
    return dtype == GLR_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void put(void* p, int64_t i, int dtype, float v) {
    if (dtype == GLR_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<float*>(p)[i] = v;
}

// One thread's elements of a 64 x 32 slab of an operand X(i, p) = x[i si + p sp], zero past its ends: vectors of 16
// bytes along the contiguous index, or, where rows are not on 16 bytes, single elements, neighbouring threads'
// next to each other (in a thread's own eight they would touch a sector for every two bytes).
template <class T>
struct Slab {
    static constexpr int V = Traits<T>::kVec, P = Traits<T>::kPitch;
    static constexpr int kPer = kTile * kSlab / V / kThreads;
    T r[kPer][V];
    __device__ __forceinline__ void load(const T* x, int64_t si, int64_t sp, int64_t i0, int64_t p0, int64_t ni, int64_t np,
                                         bool wide) {
        const bool along_p = sp == 1;
        if (wide) {
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int v = threadIdx.x + u * kThreads;
                const int64_t i = i0 + (along_p ? v / (kSlab / V) : v % (kTile / V) * V);
                const int64_t p = p0 + (along_p ? v % (kSlab / V) * V : v / (kTile / V));
                const bool in = along_p ? i < ni : p < np;
                const int64_t left = !in ? 0 : along_p ? np - p : ni - i;
                const T* src = x + i * si + p * sp;
                if (left >= V) {
                    *reinterpret_cast<uint4*>(r[u]) = *reinterpret_cast<const uint4*>(src);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) r[u][e] = e < left ? src[e] : T(0.f);
                }
            }
        } else {
            const int64_t i = i0 + (along_p ? threadIdx.x / kSlab : threadIdx.x % kTile), p = p0 + (along_p ? threadIdx.x % kSlab : threadIdx.x / kTile);
            const int64_t di = along_p ? kThreads / kSlab : 0, dp = along_p ? 0 : kThreads / kTile;
#pragma unroll
            for (int u = 0; u < kPer; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int64_t ie = i + (u * V + e) * di, pe = p + (u * V + e) * dp;
                    r[u][e] = ie < ni && pe < np ? x[ie * si + pe * sp] : T(0.f);
                }
        }
    }
    __device__ __forceinline__ void store(T* s, bool along_p, bool wide) const {
        if (!wide) {
            T* to = s + (along_p ? threadIdx.x / kSlab * P + threadIdx.x % kSlab : threadIdx.x % kTile * P + threadIdx.x / kTile);
            const int step = along_p ? kThreads / kSlab * P : kThreads / kTile;
#pragma unroll
            for (int u = 0; u < kPer; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) to[(u * V + e) * step] = r[u][e];
            return;
        }
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int v = threadIdx.x + u * kThreads;
            if (along_p) {
                *reinterpret_cast<uint4*>(s + v / (kSlab / V) * P + v % (kSlab / V) * V) = *reinterpret_cast<const uint4*>(r[u]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) s[(v % (kTile / V) * V + e) * P + v / (kTile / V)] = r[u][e];
            }
        }
    }
};

__device__ __forceinline__ uint32_t rna(float x) {
    uint32_t u;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(u) : "f"(x));
    return u;
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// The warp's 32 x 32 part of the tile, one slab.  The tensor cores truncate their sums, which would add up over a
// long contraction: a slab's products are summed there by themselves and join the total in rounded additions.
__device__ __forceinline__ void join(float (&total)[2][4][4], const float (&acc)[2][4][4]) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) total[m][n][q] += acc[m][n][q];
}
__device__ __forceinline__ void slab_mma(float (&total)[2][4][4], const __nv_bfloat16* a, const __nv_bfloat16* b, int g, int t) {
    constexpr int P = Traits<__nv_bfloat16>::kPitch;
    float acc[2][4][4] = {};
    auto at = [](const __nv_bfloat16* s, int row, int col) { return *reinterpret_cast<const uint32_t*>(s + row * P + col); };
#pragma unroll
    for (int k = 0; k < kSlab; k += 16) {
        uint32_t fa[2][4], fb[4][2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) fa[m][q] = at(a, 16 * m + g + 8 * (q & 1), k + 2 * t + 8 * (q >> 1));
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 2; ++q) fb[n][q] = at(b, 8 * n + g, k + 2 * t + 8 * q);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) mma_bf16(acc[m][n], fa[m], fb[n]);
    }
    join(total, acc);
}
// x = h + l.  CAREFUL: what would round up to infinity (the type's lowest value among it) is cut off instead, and an
// infinity is 1 and the infinity, so that it meets the other operand's high part alone: times a low part of 0, or of the
// other sign, it would be NaN.  Without it both make NaNs of all results that they enter, and product_kernel does the
// tile again with care: asking each time took 5 % of such a product (300 x 500 x 500: 14.2 us instead of 13.5 in a row of
// launches).
template <bool CAREFUL>
__device__ __forceinline__ void split(float x, uint32_t& h, uint32_t& l) {
    constexpr float kMost = 3.401162134214653e38f;    // (2 - 2^-10) 2^127
    h = rna(x);
    if (CAREFUL && fabsf(x) > kMost) h = isinf(x) ? __float_as_uint(copysignf(1.f, x)) : __float_as_uint(x) & 0xffffe000u;
    l = __float_as_uint(x - __uint_as_float(h));
}
template <bool CAREFUL = false>
__device__ __forceinline__ void slab_mma(float (&total)[2][4][4], const float* a, const float* b, int g, int t) {
    constexpr int P = Traits<float>::kPitch;
    float acc[2][4][4] = {};
#pragma unroll(CAREFUL ? 1 : kSlab / 8)
    for (int k = 0; k < kSlab; k += 8) {
        uint32_t ah[2][4], al[2][4], bh[4][2], bl[4][2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) split<CAREFUL>(a[(16 * m + g + 8 * (q & 1)) * P + k + t + 4 * (q >> 1)], ah[m][q], al[m][q]);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 2; ++q) split<CAREFUL>(b[(8 * n + g) * P + k + t + 4 * q], bh[n][q], bl[n][q]);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                mma_tf32(acc[m][n], al[m], bh[n]);
                mma_tf32(acc[m][n], ah[m], bl[n]);
                mma_tf32(acc[m][n], ah[m], bh[n]);
            }
    }
    join(total, acc);
}

__device__ __forceinline__ void finish(const Product& p, int node, int64_t i, int64_t j, float acc) {
    if (i >= p.M || j >= p.N) return;
    if (p.mode == kGradWeight) {
        put(p.outs[node], i * p.N + j, p.out_dtype, acc);
    } else if (p.mode == kForward) {
        const float z = p.bias ? acc + get(p.bias, j, p.dtype) : acc;
        float y = act_value<false>(z, p.act);
        if (p.add) y += get(p.add, i * p.ldadd + j, p.dtype);
        if (p.aux) put(p.aux, i * p.ldaux + j, p.dtype, z);
        put(p.out, i * p.ldo + j, p.dtype, y);
    } else {
        const float g = p.add ? acc + get(p.add, i * p.ldadd + j, p.dtype) : acc;
        const float d = p.pre ? g * act_slope<false>(get(p.pre, i * p.ldpre + j, p.dtype), p.act) : g;
        if (p.aux) put(p.aux, i * p.ldaux + j, p.dtype, g);
        put(p.out, i * p.ldo + j, p.dtype, d);
    }
}

__device__ __forceinline__ float peer_load(const float* p, uint32_t rank) {
    uint32_t addr;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <class T>
__global__ void __launch_bounds__(kThreads) product_kernel(const __grid_constant__ Product p, bool wide_a, bool wide_b) {
    chain_begin();
    constexpr int P = Traits<T>::kPitch, kPart = kTile + 1;
    constexpr int kSmem = 4 * kTile * P * static_cast<int>(sizeof(T)) > kTile * kPart * 4 ? 4 * kTile * P * static_cast<int>(sizeof(T)) : kTile * kPart * 4;
    __shared__ __align__(16) uint8_t smem[kSmem];
    T (*sa)[kTile * P] = reinterpret_cast<T (*)[kTile * P]>(smem);
    T (*sb)[kTile * P] = sa + 2;
    const int node = blockIdx.z, splits = gridDim.y, split = blockIdx.y;     // the splits of a tile are one cluster
    const int64_t tiles_n = (p.N + kTile - 1) / kTile;
    const int64_t i0 = blockIdx.x / tiles_n * kTile, j0 = blockIdx.x % tiles_n * kTile;
    const T* A = static_cast<const T*>(p.A) + node * p.sAb;
    const T* B = static_cast<const T*>(p.B) + node * p.sBb;
    const int warp = threadIdx.x >> 5, g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
    const int wm = (warp >> 1) * 32, wn = (warp & 1) * 32;
    float acc[2][4][4] = {};
    Slab<T> ra[2], rb[2];
    const int64_t all = (p.K + kSlab - 1) / kSlab, first = all * split / splits, last = all * (split + 1) / splits;
    auto fetch = [&](int q, int64_t s) {
        if (s >= last) return;
        ra[q].load(A, p.sAi, p.sAp, i0, s * kSlab, p.M, p.K, wide_a);
        rb[q].load(B, p.sBj, p.sBp, j0, s * kSlab, p.N, p.K, wide_b);
    };
    auto work = [&](int q, int64_t s) {
        ra[q].store(sa[q], p.sAp == 1, wide_a);
        rb[q].store(sb[q], p.sBp == 1, wide_b);
        __syncthreads();
        fetch(q, s + 2);
        slab_mma(acc, sa[q] + wm * P, sb[q] + wn * P, g, t);
    };
    fetch(0, first);
    fetch(1, first + 1);
    for (int64_t s = first; s < last; s += 2) {
        work(0, s);
        if (s + 1 < last) work(1, s + 1);
    }
    if constexpr (sizeof(T) == 4) {
        bool bad = false;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) bad = bad || isnan(acc[m][n][q]);
        if (__syncthreads_or(bad)) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[m][n][q] = 0.f;
#pragma unroll 1
            for (int64_t s = first; s < last; ++s) {
                fetch(0, s);
                ra[0].store(sa[0], p.sAp == 1, wide_a);
                rb[0].store(sb[0], p.sBp == 1, wide_b);
                __syncthreads();
                slab_mma<true>(acc, sa[0] + wm * P, sb[0] + wn * P, g, t);
                __syncthreads();
            }
        }
    }
    // (always through shared memory: an epilogue in line with each of a thread's 32 results is more code than a short
    // product has time to fetch, 54 us against 15 for 32 x 200 x 200)
    float* part = reinterpret_cast<float*>(smem);
    __syncthreads();                                  // every warp is done with the slabs
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part[(wm + 16 * m + g + 8 * (q >> 1)) * kPart + wn + 8 * n + 2 * t + (q & 1)] = acc[m][n][q];
    cluster_sync();
    const int rows = kTile / splits;                  // this CTA's rows of the tile
    for (int e = threadIdx.x; e < rows * kTile; e += kThreads) {
        const int i = split * rows + e / kTile, j = e % kTile;
        if (i0 + i >= p.M || j0 + j >= p.N) continue;
        float v = 0.f;
        for (int q = 0; q < splits; ++q) v += peer_load(part + i * kPart + j, q);
        finish(p, node, i0 + i, j0 + j, v);
    }
    cluster_sync();                                   // the peers are done with this CTA's shared memory
}

// Few rows against a matrix along the contraction (one token's forward product): the matrix is read once, in 16-byte
// loads, and the rows come from the L1 for every four of its rows.  A warp takes four results of each row, lanes along
// the contraction, its next loads in flight under the present ones' products (fp32, rounded); `ways` warps of a CTA
// share them where they would leave SMs without warps.  Lanes' sums are exchanged by halves and added up in a fixed
// order.  More than eight rows: CTAs for each eight.  Bound by HBM to four rows, by the products beyond.
// One row of 2048 x 2048 bf16 8.8 us with its launch (128 x 64 tensor-core tiles: 23), of 11008 x 4096 25 us (72), of
// 4096 x 11008 25 us (54); eight rows of the three 11, 38, 38 us (25, 64, 46).
constexpr int kRowsCols = 4, kRowsWarps = 8;
__device__ __forceinline__ void widen(const uint4& u, float (&f)[8], const __nv_bfloat16*) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) { f[2 * q] = __uint_as_float(w[q] << 16); f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const uint4& u, float (&f)[4], const float*) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
}
// Sixteen bytes past the L1.  Volatile and clobbering memory, which keeps it behind chain_begin's wait: the kernel before
// may be writing these matrices until then, and for the same reason they are not read as constant data (.nc, __ldg).
__device__ __forceinline__ uint4 load_once(const uint4* p) {
    uint4 u;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
    return u;
}
template <class T, int R>
__global__ void __launch_bounds__(kRowsWarps * 32, 2) rows_kernel(const __grid_constant__ Product p, int ways) {
    chain_begin();
    constexpr int E = 16 / static_cast<int>(sizeof(T)), C = kRowsCols, U = R <= 2 ? 2 : 1, n = R * C;
    __shared__ float part[kRowsWarps][n];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, groups = kRowsWarps / ways, way = warp % ways;
    const int64_t j0 = (static_cast<int64_t>(blockIdx.x) * groups + warp / ways) * C;
    const int64_t i0 = static_cast<int64_t>(blockIdx.y) * R;
    const T* A = static_cast<const T*>(p.A);
    const T* B = static_cast<const T*>(p.B);
    const uint4 *a[R], *b[C];                         // rows past the ends: the last one once more
#pragma unroll
    for (int r = 0; r < R; ++r) a[r] = reinterpret_cast<const uint4*>(A + min(i0 + r, p.M - 1) * p.sAi);
#pragma unroll
    for (int c = 0; c < C; ++c) b[c] = reinterpret_cast<const uint4*>(B + min(j0 + c, p.N - 1) * p.sBj);
    float sum[n];
#pragma unroll
    for (int q = 0; q < n; ++q) sum[q] = 0.f;
    const int64_t nv = p.K / E;
    const int step = 32 * ways;
    constexpr bool EARLY = R < 8;       // eight rows' vectors would not fit the registers
    uint4 next[U][C];
    auto ask = [&](int64_t v) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c) next[u][c] = v + u * step < nv ? load_once(b[c] + v + u * step) : uint4{0, 0, 0, 0};
    };
    int64_t v = way * 32 + lane;
    ask(v);
    for (; v < nv; v += U * step) {
        uint4 now[U][C], row[U][EARLY ? R : 1];
        auto row_at = [&](int u, int r) { return v + u * step < nv ? a[r][v + u * step] : uint4{0, 0, 0, 0}; };
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int c = 0; c < C; ++c) now[u][c] = next[u][c];
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (EARLY) row[u][r] = row_at(u, r);
        }
        ask(v + U * step);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float w[C][E];
#pragma unroll
            for (int c = 0; c < C; ++c) widen(now[u][c], w[c], B);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float x[E];
                widen(EARLY ? row[u][r] : row_at(u, r), x, A);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) sum[r * C + c] = fmaf(x[e], w[c][e], sum[r * C + c]);
            }
        }
    }
    // the elements past the last whole vector: a lane each
    if (const int64_t k = nv * E + lane; way == 0 && k < p.K) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c)
                sum[r * C + c] = fmaf(to_f(reinterpret_cast<const T*>(a[r])[k]), to_f(reinterpret_cast<const T*>(b[c])[k]), sum[r * C + c]);
    }
    // lanes 32 q / n .. hold the total of sum q
    int width = n;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const bool upper = lane & off;
        if (width > 1) {
            width >>= 1;
#pragma unroll
            for (int q = 0; q < n / 2; ++q)
                if (q < width) {
                    const float keep = upper ? sum[q + width] : sum[q], give = upper ? sum[q] : sum[q + width];
                    sum[q] = keep + __shfl_xor_sync(0xffffffffu, give, off);
                }
        } else {
            sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], off);
        }
    }
    if (lane % (32 / n) == 0) part[warp][lane / (32 / n)] = sum[0];
    __syncthreads();
    for (int e = threadIdx.x; e < groups * n; e += kRowsWarps * 32) {
        const int g = e / n, q = e % n;
        float v = 0.f;
        for (int w = 0; w < ways; ++w) v += part[g * ways + w][q];
        finish(p, 0, i0 + q / C, (static_cast<int64_t>(blockIdx.x) * groups + g) * C + q % C, v);
    }
}
template <class T, int R>
cudaError_t launch_rows(const Product& p, cudaStream_t st) {
    // ways to share the contraction: up to 32 warps an SM, each with two loads of a row at least (one row of 2048 x 2048 bf16
    // 10.9 -> 8.9 us, of 11008 x 4096 27 -> 25)
    constexpr int C = kRowsCols, E = 16 / static_cast<int>(sizeof(T));
    int ways = 1;
    while (ways < kRowsWarps && p.N / C * ways < 152 * 32 && p.K / E >= 128 * ways) ways *= 2;
    const int64_t per = kRowsWarps / ways * C, blocks = (p.N + per - 1) / per;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_chain(rows_kernel<T, R>, dim3(static_cast<unsigned>(blocks), static_cast<unsigned>((p.M + R - 1) / R)),
                        dim3(kRowsWarps * 32), 0, st, p, ways);
}
template <class T>
cudaError_t few_rows(const Product& p, cudaStream_t st) {
    return p.M == 1 ? launch_rows<T, 1>(p, st) : p.M == 2 ? launch_rows<T, 2>(p, st) : p.M <= 4 ? launch_rows<T, 4>(p, st) : launch_rows<T, 8>(p, st);
}

// Column sums: 64 columns a CTA, eight neighbouring ones (16 bytes of bf16) a thread and 32 rows of threads; a
// cluster of up to eight CTAs shares the rows where the columns leave SMs idle.  Added in a fixed order: down a
// thread's rows, up the rows of threads, over the cluster's CTAs.  Bound by HBM (8192 x 5632 bf16 of eight nodes: 21 us,
// 4.4 TB/s; 8192 x 1000: 10 us, without the clusters 59).
constexpr int kSumCols = 64, kSumThreads = 256, kSumLanes = kSumThreads / (kSumCols / 8);
template <class T>
__global__ void __launch_bounds__(kSumThreads) column_sums_kernel(const __grid_constant__ ColumnSums c, bool wide) {
    chain_begin();
    __shared__ float part[kSumLanes][kSumCols + 1];
    __shared__ float sums[kSumCols];
    const int node = blockIdx.z, splits = gridDim.y, split = blockIdx.y;
    const int col = threadIdx.x % (kSumCols / 8) * 8, lane = threadIdx.x / (kSumCols / 8);
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kSumCols + col;
    const int left = static_cast<int>(c.n - j < 8 ? c.n - j : 8);
    const int64_t r0 = c.rows * split / splits, r1 = c.rows * (split + 1) / splits;
    const T* x = static_cast<const T*>(c.x) + node * c.rows * c.ldx + j;
    float s[8] = {};
    if (wide && left == 8) {
        // loads of several rows at once, zero past the last one
        constexpr int kPer = 8 / Traits<T>::kVec, kAhead = 8 / kPer;
        for (int64_t i = r0 + lane; i < r1; i += kAhead * kSumLanes) {
            uint4 u[kAhead][kPer];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int h = 0; h < kPer; ++h)
                    u[q][h] = i + q * kSumLanes < r1 ? load_once(reinterpret_cast<const uint4*>(x + (i + q * kSumLanes) * c.ldx) + h) : uint4{0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int h = 0; h < kPer; ++h) {
                    float f[Traits<T>::kVec];
                    widen(u[q][h], f, static_cast<const T*>(nullptr));
#pragma unroll
                    for (int e = 0; e < Traits<T>::kVec; ++e) s[h * Traits<T>::kVec + e] += f[e];
                }
        }
    } else if (left > 0) {
        for (int64_t i = r0 + lane; i < r1; i += kSumLanes)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) s[e] += to_f(x[i * c.ldx + e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[lane][col + e] = s[e];
    __syncthreads();
    const int64_t k = static_cast<int64_t>(blockIdx.x) * kSumCols + threadIdx.x;
    if (threadIdx.x < kSumCols) {
        float v = 0.f;
        for (int q = 0; q < kSumLanes; ++q) v += part[q][threadIdx.x];
        sums[threadIdx.x] = v;
        if (splits == 1 && k < c.n) put(c.sums[node], k, c.out_dtype, v);
    }
    if (splits == 1) return;
    cluster_sync();
    if (split == 0 && threadIdx.x < kSumCols && k < c.n) {
        float v = 0.f;
        for (int q = 0; q < splits; ++q) v += peer_load(sums + threadIdx.x, q);
        put(c.sums[node], k, c.out_dtype, v);
    }
    cluster_sync();
}

// launch_chain with clusters of 1 x splits CTAs.
template <class... Q, class... A>
cudaError_t launch_clusters(void (*kernel)(Q...), dim3 grid, int threads, int splits, cudaStream_t st, const A&... args) {
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = splits; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = threads; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

int64_t any_tiles(const Product& p) { return ((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile); }
int any_splits(const Product& p) {
    // CTAs a tile: as many as fill the SMs, as long as each keeps two slabs (100 x 300 x 200 fp32 31 -> 15 us; 64 x 64 over 2000
    // rows 136 -> 23)
    const int64_t slabs = (p.K + kSlab - 1) / kSlab;
    int splits = 1;
    while (splits < 8 && any_tiles(p) * p.nodes * splits < 152 && slabs >= 4 * splits) splits *= 2;
    return splits;
}

// Sixteen-byte loads: the base, the row stride and the nodes' stride on 16 bytes.
bool wide_ok(const void* base, int64_t row_stride, int64_t node_stride, int64_t esize) {
    return reinterpret_cast<uintptr_t>(base) % 16 == 0 && row_stride * esize % 16 == 0 && node_stride * esize % 16 == 0;
}

}  // namespace

Plan plan_of(const Product& p) {
    if (p.M == 0 || p.N == 0) return {Way::kNone, {}};
    // Few rows: the tensor cores' tiles cost the same from one row to 128 (bf16 4096 x 11008: 46 us, few_rows' 25 for one row,
    // 38 for eight); fp32 ones go through any_product below 128 rows (11008 x 4096: 255 us, few_rows' 37 for one row,
    // 144 for 24).
    const int64_t es = p.dtype == GLR_BF16 ? 2 : 4;
    if (p.mode == kForward && p.M <= (p.dtype == GLR_BF16 ? 8 : 24) && p.K > 0 && p.sAp == 1 && p.sBp == 1 && wide_ok(p.A, p.M == 1 ? 0 : p.sAi, 0, es) &&
        wide_ok(p.B, p.N == 1 ? 0 : p.sBj, 0, es))
        return {Way::kFewRows, {}};
    const TcPlan tc = tc_plan(p);
    return {tc.ok ? Way::kTensorCores : Way::kAny, tc};
}

cudaError_t product(const Product& p, void* workspace, int64_t workspace_bytes, cudaStream_t st) {
    const Plan plan = plan_of(p);
    if (plan.way == Way::kNone) return cudaSuccess;
    if (plan.way == Way::kFewRows) return p.dtype == GLR_BF16 ? few_rows<__nv_bfloat16>(p, st) : few_rows<float>(p, st);
    const bool fits = plan.tc.bytes() == 0 || (workspace && workspace_bytes >= plan.tc.bytes());
    return plan.way == Way::kTensorCores && fits ? tc_product(p, plan.tc, workspace, st) : any_product(p, st);
}

cudaError_t any_product(const Product& p, cudaStream_t st) {
    const int64_t es = p.dtype == GLR_BF16 ? 2 : 4;
    const int64_t tiles = ((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile);
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    const bool wa = wide_ok(p.A, p.sAp == 1 ? p.sAi : p.sAp, p.sAb, es), wb = wide_ok(p.B, p.sBp == 1 ? p.sBj : p.sBp, p.sBb, es);
    const int splits = any_splits(p);
    const dim3 grid(static_cast<unsigned>(tiles), splits, p.nodes);
    return p.dtype == GLR_BF16 ? launch_clusters(product_kernel<__nv_bfloat16>, grid, kThreads, splits, st, p, wa, wb)
                               : launch_clusters(product_kernel<float>, grid, kThreads, splits, st, p, wa, wb);
}

// Waves of two CTAs an SM; a slab a CTA takes about 2 us, an epilogue 4 (bf16) or 7.
double any_cost(const Product& p) {
    const int splits = any_splits(p);
    const int64_t ctas = any_tiles(p) * p.nodes * splits, slabs = (p.K + kSlab - 1) / kSlab;
    const double waves = static_cast<double>((ctas + 303) / 304), mine = static_cast<double>((slabs + splits - 1) / splits);
    return 3 + waves * (p.dtype == GLR_BF16 ? 4 + 2.0 * mine : 7 + 2.4 * mine);
}

cudaError_t column_sums(const ColumnSums& c, cudaStream_t st) {
    if (c.n == 0) return cudaSuccess;
    const int64_t blocks = (c.n + kSumCols - 1) / kSumCols;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    int splits = 1;
    while (splits < 8 && blocks * c.nodes * splits < 304 && c.rows >= 256 * splits) splits *= 2;
    const bool wide = wide_ok(c.x, c.ldx, c.rows * c.ldx, c.dtype == GLR_BF16 ? 2 : 4);
    const dim3 grid(static_cast<unsigned>(blocks), splits, c.nodes);
    return c.dtype == GLR_BF16 ? launch_clusters(column_sums_kernel<__nv_bfloat16>, grid, kSumThreads, splits, st, c, wide)
                               : launch_clusters(column_sums_kernel<float>, grid, kSumThreads, splits, st, c, wide);
}

}  // namespace linear
}  // namespace glr
