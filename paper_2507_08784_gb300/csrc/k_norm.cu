// Root-mean-square norm with the residual's addition and an output in 8 bits, and its gradients.
//
// h = x + r, rstd = (mean h^2 + eps)^(-1/2), y = h rstd w: a row is read once and lies in registers, eight neighbouring
// elements a vector, up to four vectors a thread, while its squares are summed.  The squares are summed over h in 32 bits,
// before its rounding for H; where they leave the range of fp32 (h beyond 1e19) the sum is formed again of h 2^-72.
// The gradient, dx = rstd (w dy - x^ mean(w dy x^)) + d with x^ = h rstd, needs one sum a row; dw_j = sum_t dy x^ is summed by
// each CTA over its rows of one node in registers, and over the CTAs by a second kernel in their order.
// Both are bound by HBM.
#include <algorithm>

#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kMaxWarps = 32;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// The sum over the `warps` warps that share a row (in the same order for all of them); `part` is theirs until the next call
// but one.
__device__ __forceinline__ float row_sum(float v, int warps, float* part, int& turn) {
    v = warp_sum(v);
    if (warps == 1) return v;
    float* p = part + turn * kMaxWarps;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) p[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < warps ? p[threadIdx.x & 31] : 0.f;
    return warp_sum(v);
}

struct Wide { bool x, r, h, y, w, codes; };

// A row a CTA of several warps, or a row a warp (ROWS = warps of the CTA).
template <class T, int V, int MOST>
__global__ void __launch_bounds__(MOST) norm_kernel(const __grid_constant__ Norm a, Wide wide, int warps) {
    chain_begin();
    __shared__ float part[2 * kMaxWarps];
    int turn = 0;
    const int per = warps * 32, at = threadIdx.x % per;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * (blockDim.x / per) + threadIdx.x / per;
    if (i >= a.rows) return;                         // whole warps, and none waits for another one then
    const T* x = static_cast<const T*>(a.X) + i * a.ldx;
    const T* r = static_cast<const T*>(a.residual) + i * a.ldr;
    float h[V][8], ss = 0.f;
#pragma unroll
    for (int q = 0; q < V; ++q) {
        const int j = (q * per + at) * 8, n = min(8, a.n - j);
        load8(x + j, n, wide.x, h[q]);
    }
    if (a.residual) {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int j = (q * per + at) * 8, n = min(8, a.n - j);
            float d[8];
            load8(r + j, n, wide.r, d);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[q][e] += d[e];
        }
    }
#pragma unroll
    for (int q = 0; q < V; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(h[q][e], h[q][e], ss);
    ss = row_sum(ss, warps, part, turn);
    float rstd = 1.f / sqrtf(ss / static_cast<float>(a.n) + a.eps);
    if (ss > 3.0e38f) {
        constexpr float kDown = 2.117582368135751e-22f;      // 2^-72: 32768 of fp32's largest squares stay in its range
        float low = 0.f;
#pragma unroll
        for (int q = 0; q < V; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) { const float y = h[q][e] * kDown; low = fmaf(y, y, low); }
        low = row_sum(low, warps, part, turn);
        rstd = kDown / sqrtf(low / static_cast<float>(a.n));
    }
    if (a.rstd && at == 0) a.rstd[i] = rstd;
#pragma unroll
    for (int q = 0; q < V; ++q) {
        const int j = (q * per + at) * 8, n = min(8, a.n - j);
        if (a.H) store8(static_cast<T*>(a.H) + i * a.ldh + j, n, wide.h, h[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[q][e] *= rstd;
        if (a.weight) {
            float w[8];
            load8(static_cast<const T*>(a.weight) + j, n, wide.w, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[q][e] *= w[e];
        }
        if (a.Y) store8(static_cast<T*>(a.Y) + i * a.ldy + j, n, wide.y, h[q]);
        if (a.codes) {
            const uint32_t s = block_scale(h[q]);
            const uint2 c = block_codes(h[q], s);
            if (n > 0) {
                store_codes(a.codes + i * a.ld_codes + j, n, wide.codes, c);
                if ((at & 3) == 0) a.scales[i * a.ld_scales + j / kBlock] = static_cast<uint8_t>(s);
            }
        }
    }
}

// CTA b of a node takes the node's rows [rows b / blocks, rows (b + 1) / blocks); where a row is a warp's, its warps take them in
// turn and add up their sums at the end.
template <class T, int V, int MOST>
__global__ void __launch_bounds__(MOST) norm_grad_kernel(const __grid_constant__ NormGrad a, Wide wide, int warps) {
    chain_begin();
    __shared__ float part[2 * kMaxWarps];
    extern __shared__ float sums[];                  // a row's columns, where several of the CTA's rows have sums of their own
    int turn = 0;
    const int per = warps * 32, at = threadIdx.x % per, groups = blockDim.x / per, group = threadIdx.x / per;
    const int64_t node = blockIdx.y, blocks = gridDim.x, b = blockIdx.x;
    const int64_t r0 = node * a.rows + a.rows * b / blocks, r1 = node * a.rows + a.rows * (b + 1) / blocks;
    const float share = 1.f / static_cast<float>(a.n);
    float dw[V][8];
#pragma unroll
    for (int q = 0; q < V; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[q][e] = 0.f;
    for (int64_t i = r0 + group; i < r1; i += groups) {
        const T* dy = static_cast<const T*>(a.dY) + i * a.lddy;
        const T* h = static_cast<const T*>(a.H) + i * a.ldh;
        const float rstd = a.rstd[i];
        float x[V][8], g[V][8], dot = 0.f;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int j = (q * per + at) * 8, n = min(8, a.n - j);
            load8(dy + j, n, wide.y, g[q]);
            load8(h + j, n, wide.h, x[q]);
        }
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int j = (q * per + at) * 8, n = min(8, a.n - j);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[q][e] *= rstd;
                dw[q][e] = fmaf(g[q][e], x[q][e], dw[q][e]);
            }
            if (a.weight) {
                float w[8];
                load8(static_cast<const T*>(a.weight) + j, n, wide.w, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[q][e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) dot = fmaf(g[q][e], x[q][e], dot);
        }
        dot = row_sum(dot, warps, part, turn) * share;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int j = (q * per + at) * 8, n = min(8, a.n - j);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[q][e] = rstd * (g[q][e] - x[q][e] * dot);
            if (a.residual) {
                float d[8];
                load8(static_cast<const T*>(a.residual) + i * a.ldr + j, n, wide.r, d);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[q][e] += d[e];
            }
            if (a.dX) store8(static_cast<T*>(a.dX) + i * a.lddx + j, n, wide.x, g[q]);
        }
    }
    if (!a.want_dweight) return;
    float* to = a.partial + (node * blocks + b) * a.n;
    if (groups == 1) {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int j = (q * per + at) * 8, n = min(8, a.n - j);
            store8(to + j, n, a.n % 4 == 0, dw[q]);
        }
        return;
    }
    for (int k = 0; k < groups; ++k) {               // one group after the other: a fixed order
        if (k == group)
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const int j = (q * per + at) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + e < a.n) sums[j + e] = k ? sums[j + e] + dw[q][e] : dw[q][e];
            }
        __syncthreads();
    }
    for (int j = threadIdx.x; j < a.n; j += blockDim.x) to[j] = sums[j];
}

// dweight[node][j] = the sum of the node's partial sums, in their order; 32 columns a CTA, eight warps sharing them.
constexpr int kSumThreads = 256;
template <class G>
__global__ void __launch_bounds__(kSumThreads) norm_sum_kernel(const __grid_constant__ NormGrad a, int blocks) {
    chain_begin();
    __shared__ float part[kSumThreads / 32][33];
    const int64_t node = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (j < a.n)
        for (int b = warp; b < blocks; b += kSumThreads / 32) v += a.partial[(node * blocks + b) * a.n + j];
    part[warp][lane] = v;
    __syncthreads();
    if (warp || j >= a.n) return;
    for (int w = 1; w < kSumThreads / 32; ++w) v += part[w][lane];
    put(static_cast<G*>(a.dweight[node]) + j, v);
}

bool on16(const void* p, int64_t ld_bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld_bytes % 16 == 0; }

// Warps a row and vectors a thread: a warp up to 1024 columns, more where a thread would have over four vectors.
struct Shape { int warps, vectors, threads; };
Shape shape_of(int n) {
    int warps = 1;
    if (n > 1024) {
        warps = 4;
        while (warps < 32 && n > warps * 32 * 16) warps *= 2;
    }
    const int v = (n + warps * 256 - 1) / (warps * 256);
    return {warps, v <= 1 ? 1 : v <= 2 ? 2 : 4, warps == 1 ? 256 : warps * 32};
}

// CTAs a node of the gradient's kernel: enough for every SM's threads, each with a row at least.
int64_t grad_blocks(int64_t nodes, int64_t rows, int n) {
    const Shape s = shape_of(n);
    const int64_t groups = s.threads / (s.warps * 32), most = std::max<int64_t>(1, 152 * (1024 / s.threads) / nodes);
    return std::max<int64_t>(1, std::min(most, (rows + groups - 1) / groups));
}

// kernel<vectors, most threads> by a row's shape (a warp's four vectors are those of 256 threads)
#define GLR_BY_SHAPE(kernel, T)                                                                                     \
    (s.threads <= 256 ? (s.vectors == 1 ? kernel<T, 1, 256> : s.vectors == 2 ? kernel<T, 2, 256> : kernel<T, 4, 256>) \
     : s.threads <= 512 ? (s.vectors == 1 ? kernel<T, 1, 512> : kernel<T, 2, 512>)                                   \
                        : (s.vectors == 1 ? kernel<T, 1, 1024> : s.vectors == 2 ? kernel<T, 2, 1024> : kernel<T, 4, 1024>))

template <class T>
cudaError_t launch_norm(const Norm& a, const Wide& w, cudaStream_t st) {
    const Shape s = shape_of(a.n);
    const int64_t groups = s.threads / (s.warps * 32), blocks = (a.rows + groups - 1) / groups;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_chain(GLR_BY_SHAPE(norm_kernel, T), dim3(static_cast<unsigned>(blocks)), s.threads, 0, st, a, w, s.warps);
}
template <class T>
cudaError_t launch_grad(const NormGrad& a, const Wide& w, int64_t blocks, cudaStream_t st) {
    const Shape s = shape_of(a.n);
    return launch_chain(GLR_BY_SHAPE(norm_grad_kernel, T), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.nodes)), s.threads,
                        s.warps == 1 ? a.n * sizeof(float) : 0, st, a, w, s.warps);
}

}  // namespace

cudaError_t norm(const Norm& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, several = a.rows > 1;
    const Wide w{on16(a.X, several * a.ldx * es), on16(a.residual, several * a.ldr * es), on16(a.H, several * a.ldh * es),
                 on16(a.Y, several * a.ldy * es), on16(a.weight, 0),
                 reinterpret_cast<uintptr_t>(a.codes) % 8 == 0 && several * a.ld_codes % 8 == 0};
    return dtype == GLR_BF16 ? launch_norm<__nv_bfloat16>(a, w, st) : launch_norm<float>(a, w, st);
}

int64_t norm_grad_bytes(int64_t nodes, int64_t rows, int n) { return nodes * grad_blocks(nodes, rows, n) * n * 4; }

cudaError_t norm_grad(const NormGrad& a, int dtype, int grad_dtype, cudaStream_t st) {
    if (a.rows == 0 && !a.want_dweight) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, several = a.nodes * a.rows > 1;
    const Wide w{on16(a.dX, several * a.lddx * es), on16(a.residual, several * a.ldr * es), on16(a.H, several * a.ldh * es),
                 on16(a.dY, several * a.lddy * es), on16(a.weight, 0), false};
    const int64_t blocks = grad_blocks(a.nodes, a.rows, a.n);
    cudaError_t e = dtype == GLR_BF16 ? launch_grad<__nv_bfloat16>(a, w, blocks, st) : launch_grad<float>(a, w, blocks, st);
    if (e != cudaSuccess || !a.want_dweight) return e;
    const dim3 grid((a.n + 31) / 32, static_cast<unsigned>(a.nodes));
    return grad_dtype == GLR_BF16 ? launch_chain(norm_sum_kernel<__nv_bfloat16>, grid, kSumThreads, 0, st, a, static_cast<int>(blocks))
                                  : launch_chain(norm_sum_kernel<float>, grid, kSumThreads, 0, st, a, static_cast<int>(blocks));
}

}  // namespace rows
}  // namespace glr
