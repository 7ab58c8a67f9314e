// Products of linear layers with their epilogues, for any sizes, strides and alignment: 64 x 64 output
// tiles by four warps, operand slabs of 32 contraction elements through registers into shared memory, two
// slabs deep.  bf16 operands go through mma.sync.m16n8k16; fp32 ones through m16n8k8 in the 3xTF32 form
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

// One thread's vectors of a 64 x 32 slab of an operand X(i, p) = x[i si + p sp], zero past its ends.
template <class T>
struct Slab {
    static constexpr int V = Traits<T>::kVec, P = Traits<T>::kPitch;
    static constexpr int kPer = kTile * kSlab / V / kThreads;
    T r[kPer][V];
    __device__ __forceinline__ void load(const T* x, int64_t si, int64_t sp, int64_t i0, int64_t p0, int64_t ni, int64_t np,
                                         bool wide) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int v = threadIdx.x + u * kThreads;
            // vectors run along the contiguous index
            const bool along_p = sp == 1;
            const int64_t i = i0 + (along_p ? v / (kSlab / V) : v % (kTile / V) * V);
            const int64_t p = p0 + (along_p ? v % (kSlab / V) * V : v / (kTile / V));
            const bool in = along_p ? i < ni : p < np;
            const int64_t left = !in ? 0 : along_p ? np - p : ni - i;
            const T* src = x + i * si + p * sp;
            if (wide && left >= V) {
                *reinterpret_cast<uint4*>(r[u]) = *reinterpret_cast<const uint4*>(src);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) r[u][e] = e < left ? src[e] : T(0.f);
            }
        }
    }
    __device__ __forceinline__ void store(T* s, bool along_p) const {
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

// The warp's 32 x 32 part of the tile, one slab.
__device__ __forceinline__ void slab_mma(float (&acc)[2][4][4], const __nv_bfloat16* a, const __nv_bfloat16* b, int g, int t) {
    constexpr int P = Traits<__nv_bfloat16>::kPitch;
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
}
// fp32: the tensor core truncates its sums, which would add up over a long contraction; a slab's products
// are summed there by themselves and join the total in a rounded addition.
__device__ __forceinline__ void slab_mma(float (&total)[2][4][4], const float* a, const float* b, int g, int t) {
    constexpr int P = Traits<float>::kPitch;
    float acc[2][4][4] = {};
#pragma unroll
    for (int k = 0; k < kSlab; k += 8) {
        uint32_t ah[2][4], al[2][4], bh[4][2], bl[4][2];
        auto split = [](float x, uint32_t& h, uint32_t& l) {
            h = rna(x);
            l = __float_as_uint(x - __uint_as_float(h));
        };
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) split(a[(16 * m + g + 8 * (q & 1)) * P + k + t + 4 * (q >> 1)], ah[m][q], al[m][q]);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 2; ++q) split(b[(8 * n + g) * P + k + t + 4 * q], bh[n][q], bl[n][q]);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                mma_tf32(acc[m][n], al[m], bh[n]);
                mma_tf32(acc[m][n], ah[m], bl[n]);
                mma_tf32(acc[m][n], ah[m], bh[n]);
            }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) total[m][n][q] += acc[m][n][q];
}

__device__ __forceinline__ void finish(const Product& p, int node, int64_t i, int64_t j, float acc) {
    if (i >= p.M || j >= p.N) return;
    if (p.mode == kGradWeight) {
        put(p.outs[node], i * p.N + j, p.out_dtype, acc);
    } else if (p.mode == kForward) {
        const float z = p.bias ? acc + get(p.bias, j, p.dtype) : acc;
        float y = act_value(z, p.act);
        if (p.add) y += get(p.add, i * p.ldadd + j, p.dtype);
        if (p.aux) put(p.aux, i * p.ldaux + j, p.dtype, z);
        put(p.out, i * p.ldo + j, p.dtype, y);
    } else {
        const float g = p.add ? acc + get(p.add, i * p.ldadd + j, p.dtype) : acc;
        const float d = p.pre ? g * act_slope(get(p.pre, i * p.ldpre + j, p.dtype), p.act) : g;
        if (p.aux) put(p.aux, i * p.ldaux + j, p.dtype, g);
        put(p.out, i * p.ldo + j, p.dtype, d);
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) product_kernel(const __grid_constant__ Product p, bool wide_a, bool wide_b) {
    chain_begin();
    constexpr int P = Traits<T>::kPitch;
    __shared__ __align__(16) T sa[2][kTile * P], sb[2][kTile * P];
    const int node = blockIdx.z;
    const int64_t tiles_n = (p.N + kTile - 1) / kTile;
    const int64_t i0 = blockIdx.x / tiles_n * kTile, j0 = blockIdx.x % tiles_n * kTile;
    const T* A = static_cast<const T*>(p.A) + node * p.sAb;
    const T* B = static_cast<const T*>(p.B) + node * p.sBb;
    const int warp = threadIdx.x >> 5, g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
    const int wm = (warp >> 1) * 32, wn = (warp & 1) * 32;
    float acc[2][4][4] = {};
    Slab<T> ra, rb;
    const int64_t slabs = (p.K + kSlab - 1) / kSlab;
    if (slabs > 0) {
        ra.load(A, p.sAi, p.sAp, i0, 0, p.M, p.K, wide_a);
        rb.load(B, p.sBj, p.sBp, j0, 0, p.N, p.K, wide_b);
    }
    for (int64_t s = 0; s < slabs; ++s) {
        const int buf = s & 1;
        ra.store(sa[buf], p.sAp == 1);
        rb.store(sb[buf], p.sBp == 1);
        __syncthreads();
        if (s + 1 < slabs) {
            ra.load(A, p.sAi, p.sAp, i0, (s + 1) * kSlab, p.M, p.K, wide_a);
            rb.load(B, p.sBj, p.sBp, j0, (s + 1) * kSlab, p.N, p.K, wide_b);
        }
        slab_mma(acc, sa[buf] + wm * P, sb[buf] + wn * P, g, t);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                finish(p, node, i0 + wm + 16 * m + g + 8 * (q >> 1), j0 + wn + 8 * n + 2 * t + (q & 1), acc[m][n][q]);
}

// 32 columns a CTA, eight rows of threads down them; the eight sums are added in order.
constexpr int kSumCols = 32, kSumRows = 8;
__global__ void __launch_bounds__(kSumCols * kSumRows) column_sums_kernel(const __grid_constant__ ColumnSums c) {
    chain_begin();
    __shared__ float part[kSumRows][kSumCols];
    const int node = blockIdx.y, tx = threadIdx.x % kSumCols, ty = threadIdx.x / kSumCols;
    const int64_t j = static_cast<int64_t>(blockIdx.x) * kSumCols + tx;
    float s = 0.f;
    if (j < c.n)
        for (int64_t i = ty; i < c.rows; i += kSumRows) s += get(c.x, (node * c.rows + i) * c.ldx + j, c.dtype);
    part[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && j < c.n) {
        for (int y = 1; y < kSumRows; ++y) s += part[y][tx];
        put(c.sums[node], j, c.out_dtype, s);
    }
}

// Sixteen-byte loads: the base, the row stride and the nodes' stride on 16 bytes.
bool wide_ok(const void* base, int64_t row_stride, int64_t node_stride, int64_t esize) {
    return reinterpret_cast<uintptr_t>(base) % 16 == 0 && row_stride * esize % 16 == 0 && node_stride * esize % 16 == 0;
}

}  // namespace

cudaError_t product(const Product& p, cudaStream_t st) {
    if (p.M == 0 || p.N == 0) return cudaSuccess;
    return tc_ok(p) ? tc_product(p, st) : any_product(p, st);
}

cudaError_t any_product(const Product& p, cudaStream_t st) {
    const int64_t es = p.dtype == GLR_BF16 ? 2 : 4;
    const int64_t tiles = ((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile);
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    const bool wa = wide_ok(p.A, p.sAp == 1 ? p.sAi : p.sAp, p.sAb, es), wb = wide_ok(p.B, p.sBp == 1 ? p.sBj : p.sBp, p.sBb, es);
    const dim3 grid(static_cast<unsigned>(tiles), 1, p.nodes);
    return p.dtype == GLR_BF16 ? launch_chain(product_kernel<__nv_bfloat16>, grid, kThreads, 0, st, p, wa, wb)
                               : launch_chain(product_kernel<float>, grid, kThreads, 0, st, p, wa, wb);
}

cudaError_t column_sums(const ColumnSums& c, cudaStream_t st) {
    if (c.n == 0) return cudaSuccess;
    const int64_t blocks = (c.n + kSumCols - 1) / kSumCols;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_chain(column_sums_kernel, dim3(static_cast<unsigned>(blocks), c.nodes), kSumCols * kSumRows, 0, st, c);
}

}  // namespace linear
}  // namespace glr
