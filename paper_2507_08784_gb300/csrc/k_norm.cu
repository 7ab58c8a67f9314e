// Root-mean-square norm with the residual's addition and an output in 8 bits, and its gradients.
//
// h = x + r, rstd = (mean h^2 + eps)^(-1/2), y = h rstd w: a row is read once and lies in registers while its squares are summed.
// They are summed over h in 32 bits, before its rounding for H (one rounding a result); where they leave the range of fp32
// (h beyond 1e19) the sum is formed again of h 2^-72.
// The gradient, dx = rstd (w dy - x^ mean(w dy x^)) + d with x^ = h rstd, needs one sum a row; dw_j = sum_t dy x^ is summed by
// each CTA over its rows of one node in registers, and over the CTAs by a second kernel in their order.
// Both are bound by HBM: 8192 x 4096 bf16 with residual and 8-bit output 54 us (303 MB, 5.6 TB/s), gradient of eight nodes with
// residual 57 us (268 MB, 4.7 TB/s), 4 of them the second kernel's.  A row a CTA at a time, without the ring of rows on their way,
// took 72 and 122.
#include <algorithm>

#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kMaxWarps = 32;
constexpr float kDown = 2.117582368135751e-22f;      // 2^-72: 32768 of fp32's largest squares stay in its range

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

// Rows off 16 bytes, or too long for the ring kernels below: a row a warp, or a CTA of several warps; each lane's eight columns
// of a warp's 256 are 32 apart.
template <class T, int V, int MOST>
__global__ void __launch_bounds__(MOST) norm_kernel(const __grid_constant__ Norm a, int warps, bool wide_codes) {
    chain_begin();
    __shared__ __align__(16) float turned[MOST / 32][256];
    __shared__ float part[2 * kMaxWarps];
    int turn = 0;
    const int per = warps * 32, at = threadIdx.x % per, warp = at >> 5;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * (blockDim.x / per) + threadIdx.x / per;
    if (i >= a.rows) return;                         // whole warps, and none waits for another one then
    float h[V][8], ss = 0.f;
#pragma unroll
    for (int q = 0; q < V; ++q) load_apart(static_cast<const T*>(a.X) + i * a.ldx, (q * warps + warp) * 256, a.n, h[q]);
    if (a.residual) {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            float d[8];
            load_apart(static_cast<const T*>(a.residual) + i * a.ldr, (q * warps + warp) * 256, a.n, d);
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
        const int first = (q * warps + warp) * 256;
        if (a.H) store_apart(static_cast<T*>(a.H) + i * a.ldh, first, a.n, h[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[q][e] *= rstd;
        if (a.weight) {
            float w[8];
            load_apart(static_cast<const T*>(a.weight), first, a.n, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[q][e] *= w[e];
        }
        if (a.Y) store_apart(static_cast<T*>(a.Y) + i * a.ldy, first, a.n, h[q]);
        if (a.codes) store_blocks(a.codes + i * a.ld_codes, a.scales + i * a.ld_scales, first, a.n, wide_codes, h[q], turned[threadIdx.x >> 5]);
    }
}

// CTA b of a node takes the node's rows [rows b / blocks, rows (b + 1) / blocks); where a row is a warp's, its warps take them in
// turn and add up their sums at the end.
template <class T, int V, int MOST>
__global__ void __launch_bounds__(MOST) norm_grad_kernel(const __grid_constant__ NormGrad a, int warps) {
    chain_begin();
    __shared__ float part[2 * kMaxWarps];
    extern __shared__ float sums[];                  // a row's columns, where several of the CTA's rows have sums of their own
    int turn = 0;
    const int per = warps * 32, warp = threadIdx.x % per >> 5, lane = threadIdx.x & 31, groups = blockDim.x / per, group = threadIdx.x / per;
    const int64_t node = blockIdx.y, blocks = gridDim.x, b = blockIdx.x;
    const int64_t r0 = node * a.rows + a.rows * b / blocks, r1 = node * a.rows + a.rows * (b + 1) / blocks;
    const float share = 1.f / static_cast<float>(a.n);
    float dw[V][8];
#pragma unroll
    for (int q = 0; q < V; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[q][e] = 0.f;
    for (int64_t i = r0 + group; i < r1; i += groups) {
        const float rstd = a.rstd[i];
        float x[V][8], g[V][8], dot = 0.f;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            load_apart(static_cast<const T*>(a.dY) + i * a.lddy, (q * warps + warp) * 256, a.n, g[q]);
            load_apart(static_cast<const T*>(a.H) + i * a.ldh, (q * warps + warp) * 256, a.n, x[q]);
        }
#pragma unroll
        for (int q = 0; q < V; ++q) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[q][e] *= rstd;
                dw[q][e] = fmaf(g[q][e], x[q][e], dw[q][e]);
            }
            if (a.weight) {
                float w[8];
                load_apart(static_cast<const T*>(a.weight), (q * warps + warp) * 256, a.n, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[q][e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) dot = fmaf(g[q][e], x[q][e], dot);
        }
        dot = row_sum(dot, warps, part, turn) * share;
        if (!a.dX) continue;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int first = (q * warps + warp) * 256;
#pragma unroll
            for (int e = 0; e < 8; ++e) g[q][e] = rstd * (g[q][e] - x[q][e] * dot);
            if (a.residual) {
                float d[8];
                load_apart(static_cast<const T*>(a.residual) + i * a.ldr, first, a.n, d);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[q][e] += d[e];
            }
            store_apart(static_cast<T*>(a.dX) + i * a.lddx, first, a.n, g[q]);
        }
    }
    if (!a.want_dweight) return;
    float* to = a.partial + (node * blocks + b) * a.n;
    if (groups == 1) {
#pragma unroll
        for (int q = 0; q < V; ++q) store_apart(to, (q * warps + warp) * 256, a.n, dw[q]);
        return;
    }
    for (int k = 0; k < groups; ++k) {               // one group after the other: a fixed order
        if (k == group)
#pragma unroll
            for (int q = 0; q < V; ++q)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = (q * warps + warp) * 256 + e * 32 + lane;
                    if (j < a.n) sums[j] = k ? sums[j] + dw[q][e] : dw[q][e];
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
#pragma unroll 8
        for (int b = warp; b < blocks; b += kSumThreads / 32) v += a.partial[(node * blocks + b) * a.n + j];
    part[warp][lane] = v;
    __syncthreads();
    if (warp || j >= a.n) return;
    for (int w = 1; w < kSumThreads / 32; ++w) v += part[w][lane];
    put(static_cast<G*>(a.dweight[node]) + j, v);
}

// ---- rows on 16 bytes ---------------------------------------------------------------------------------------------
// A CTA goes through several rows, the next two on their way by asynchronous copies meanwhile: each thread copies what it
// will read itself, so that a copy is only waited for by its thread.  Sixteen columns a thread, in chunks of 16 bytes.
// Three stages, or two where three do not fit.
constexpr size_t kRingBytes = 200 * 1024;
template <class T, int NT, int MATRICES> constexpr int kStages = size_t(3) * MATRICES * 16 * sizeof(T) * NT > kRingBytes ? 2 : 3;
template <class T> constexpr int kChunks = sizeof(T) == 2 ? 2 : 4;
template <class T> constexpr int kElems = 16 / sizeof(T);

__device__ __forceinline__ uint32_t smem_at(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void copy16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_at(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until all but the last S - 2 groups are there
template <int S>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory"); }

template <class T> __device__ __forceinline__ void widen(const uint4& u, float (&v)[kElems<T>]);
template <> __device__ __forceinline__ void widen<__nv_bfloat16>(const uint4& u, float (&v)[8]) { widen8(u, v); }
template <> __device__ __forceinline__ void widen<float>(const uint4& u, float (&v)[4]) {
    v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
}
template <class T> __device__ __forceinline__ uint4 narrow(const float (&v)[kElems<T>]);
template <> __device__ __forceinline__ uint4 narrow<__nv_bfloat16>(const float (&v)[8]) {
    return make_uint4(narrow2(v[0], v[1]), narrow2(v[2], v[3]), narrow2(v[4], v[5]), narrow2(v[6], v[7]));
}
template <> __device__ __forceinline__ uint4 narrow<float>(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

// A chunk in 8 bits: 32 / E neighbouring lanes hold a block.
template <int E>
__device__ __forceinline__ void pack_chunk(const Norm& a, int64_t i, int j, const float (&v)[E]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 32 / E; o *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const uint32_t s = scale_of(m);
    if (j >= a.n) return;
    int8_t* to = a.codes + i * a.ld_codes + j;
    uint32_t w[E / 4];
#pragma unroll
    for (int h = 0; h < E / 4; ++h) w[h] = four_codes(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3], s);
    if (reinterpret_cast<uintptr_t>(to) % E == 0) {
        if (E == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[E / 4 - 1]);
        else *reinterpret_cast<uint32_t*>(to) = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = static_cast<int8_t>(w[e / 4] >> (8 * (e % 4)));
    }
    if (j % kBlock == 0) a.scales[i * a.ld_scales + j / kBlock] = static_cast<uint8_t>(s);
}

template <class T, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) norm_ring_kernel(const __grid_constant__ Norm a) {
    chain_begin();
    constexpr int K = kChunks<T>, E = kElems<T>, W = NT / 32, S = kStages<T, NT, 2>;
    extern __shared__ uint4 ring[];                  // [stage][X, residual][chunk][thread]
    __shared__ float part[2 * kMaxWarps];
    int turn = 0;
    const int tid = threadIdx.x;
    const auto at = [&](int stage, int matrix, int k) { return ring + ((stage * 2 + matrix) * K + k) * NT + tid; };
    const auto fetch = [&](int64_t i, int stage) {
        if (i < a.rows) {
            const T* x = static_cast<const T*>(a.X) + i * a.ldx;
            const T* r = static_cast<const T*>(a.residual) + i * a.ldr;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int j = (k * NT + tid) * E;
                if (j < a.n) {
                    copy16(at(stage, 0, k), x + j);
                    if (a.residual) copy16(at(stage, 1, k), r + j);
                }
            }
        }
        copies_end();
    };
    uint4 weight[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int j = (k * NT + tid) * E;
        weight[k] = a.weight && j < a.n ? reinterpret_cast<const uint4*>(static_cast<const T*>(a.weight) + j)[0] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int s = 0; s < S - 1; ++s) fetch(blockIdx.x + static_cast<int64_t>(s) * gridDim.x, s);
    int stage = 0;
    for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        copies_wait<S>();
        float h[K][E], ss = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int j = (k * NT + tid) * E;
            widen<T>(j < a.n ? *at(stage, 0, k) : make_uint4(0, 0, 0, 0), h[k]);
            if (a.residual) {
                float r[E];
                widen<T>(j < a.n ? *at(stage, 1, k) : make_uint4(0, 0, 0, 0), r);
#pragma unroll
                for (int e = 0; e < E; ++e) h[k][e] += r[e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(h[k][e], h[k][e], ss);
        }
        ss = row_sum(ss, W, part, turn);
        // the stage before this one has been read by all
        fetch(i + (S - 1) * static_cast<int64_t>(gridDim.x), stage == 0 ? S - 1 : stage - 1);
        stage = stage == S - 1 ? 0 : stage + 1;
        float rstd = 1.f / sqrtf(ss / static_cast<float>(a.n) + a.eps);
        if (ss > 3.0e38f) {
            float low = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) { const float y = h[k][e] * kDown; low = fmaf(y, y, low); }
            low = row_sum(low, W, part, turn);
            rstd = kDown / sqrtf(low / static_cast<float>(a.n));
        }
        if (a.rstd && tid == 0) a.rstd[i] = rstd;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int j = (k * NT + tid) * E;
            if (a.H && j < a.n) *reinterpret_cast<uint4*>(static_cast<T*>(a.H) + i * a.ldh + j) = narrow<T>(h[k]);
            float w[E];
            widen<T>(weight[k], w);
#pragma unroll
            for (int e = 0; e < E; ++e) { h[k][e] *= rstd; if (a.weight) h[k][e] *= w[e]; }
            if (a.Y && j < a.n) *reinterpret_cast<uint4*>(static_cast<T*>(a.Y) + i * a.ldy + j) = narrow<T>(h[k]);
            if (a.codes) pack_chunk<E>(a, i, j, h[k]);
        }
    }
}

template <class T, int NT>
__global__ void __launch_bounds__(NT, NT >= 512 ? 1024 / NT : 768 / NT) norm_grad_ring_kernel(const __grid_constant__ NormGrad a) {
    chain_begin();
    constexpr int K = kChunks<T>, E = kElems<T>, W = NT / 32, S = kStages<T, NT, 3>;
    extern __shared__ uint4 ring[];                  // [stage][dY, H, residual][chunk][thread]
    __shared__ float part[2 * kMaxWarps];
    __shared__ float rstds[S][W];
    int turn = 0;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t node = blockIdx.y, blocks = gridDim.x, b = blockIdx.x;
    const int64_t r0 = node * a.rows + a.rows * b / blocks, r1 = node * a.rows + a.rows * (b + 1) / blocks;
    const float share = 1.f / static_cast<float>(a.n);
    const auto at = [&](int stage, int matrix, int k) { return ring + ((stage * 3 + matrix) * K + k) * NT + tid; };
    const auto fetch = [&](int64_t i, int stage) {
        if (i < r1) {
            const T* y = static_cast<const T*>(a.dY) + i * a.lddy;
            const T* h = static_cast<const T*>(a.H) + i * a.ldh;
            const T* r = static_cast<const T*>(a.residual) + i * a.ldr;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int j = (k * NT + tid) * E;
                if (j < a.n) {
                    copy16(at(stage, 0, k), y + j);
                    copy16(at(stage, 1, k), h + j);
                    if (a.residual && a.dX) copy16(at(stage, 2, k), r + j);
                }
            }
            if (lane == 0) copy4(&rstds[stage][warp], a.rstd + i);
        }
        copies_end();
    };
    uint4 weight[K];
    float dw[K][E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int j = (k * NT + tid) * E;
        weight[k] = a.weight && j < a.n ? reinterpret_cast<const uint4*>(static_cast<const T*>(a.weight) + j)[0] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < E; ++e) dw[k][e] = 0.f;
    }
#pragma unroll
    for (int s = 0; s < S - 1; ++s) fetch(r0 + s, s);
    int stage = 0;
    for (int64_t i = r0; i < r1; ++i) {
        copies_wait<S>();
        __syncwarp();                                // lane 0's copy is all lanes' now
        const float rstd = rstds[stage][warp];
        float dot = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if ((k * NT + tid) * E >= a.n) continue;
            float g[E], x[E], w[E];
            widen<T>(*at(stage, 0, k), g);
            widen<T>(*at(stage, 1, k), x);
            widen<T>(weight[k], w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] *= rstd;
                dw[k][e] = fmaf(g[e], x[e], dw[k][e]);
                dot = fmaf(a.weight ? g[e] * w[e] : g[e], x[e], dot);
            }
        }
        dot = row_sum(dot, W, part, turn) * share;
        if (W == 1) __syncwarp();
        // the stage before this one has been read by all
        fetch(i + S - 1, stage == 0 ? S - 1 : stage - 1);
        if (a.dX) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int j = (k * NT + tid) * E;
                if (j >= a.n) continue;
                float g[E], x[E], w[E];
                widen<T>(*at(stage, 0, k), g);
                widen<T>(*at(stage, 1, k), x);
                widen<T>(weight[k], w);
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] = rstd * ((a.weight ? g[e] * w[e] : g[e]) - x[e] * rstd * dot);
                if (a.residual) {
                    widen<T>(*at(stage, 2, k), w);
#pragma unroll
                    for (int e = 0; e < E; ++e) g[e] += w[e];
                }
                *reinterpret_cast<uint4*>(static_cast<T*>(a.dX) + i * a.lddx + j) = narrow<T>(g);
            }
        }
        stage = stage == S - 1 ? 0 : stage + 1;
    }
    if (!a.want_dweight) return;
    float* to = a.partial + (node * blocks + b) * a.n;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int j = (k * NT + tid) * E;
        if (j < a.n)
#pragma unroll
            for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(to + j + e) = make_float4(dw[k][e], dw[k][e + 1], dw[k][e + 2], dw[k][e + 3]);
    }
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

// CTAs a node of the gradient's kernels: enough for every SM, each with a row at least.
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

// The ring kernels' threads a row, and the CTAs that an SM holds (0: their rows do not fit).
int ring_threads(int n) {
    int t = 32;
    while (t * 16 < n) t *= 2;
    return t;
}
size_t ring_bytes(int threads, int matrices, int64_t es) {
    const size_t stage = static_cast<size_t>(matrices * 16 * es) * threads;
    return 3 * stage > kRingBytes ? 2 * stage : 3 * stage;
}
int ring_ctas(int n, int matrices, int64_t es) {
    const int threads = ring_threads(n);
    if (threads > 1024 || ring_bytes(threads, matrices, es) > kRingBytes) return 0;
    const int regs = matrices == 3 && threads < 512 ? 768 / threads : 1024 / threads;
    return std::min({regs, static_cast<int>(kRingBytes / ring_bytes(threads, matrices, es)), 32});
}
template <class Kernel, class Args>
cudaError_t launch_ring(Kernel kernel, const Args& a, dim3 grid, int threads, size_t smem, cudaStream_t st) {
    if (smem > 40 * 1024) {                          // with the static part, more than a launch may have unasked
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return e;
    }
    return launch_chain(kernel, grid, threads, smem, st, a);
}
#define GLR_BY_THREADS(kernel, T, t)                                                                       \
    ((t) == 32 ? kernel<T, 32> : (t) == 64 ? kernel<T, 64> : (t) == 128 ? kernel<T, 128> : (t) == 256 ? kernel<T, 256> \
     : (t) == 512 ? kernel<T, 512> : kernel<T, 1024>)

template <class T>
cudaError_t launch_norm(const Norm& a, cudaStream_t st) {
    const Shape s = shape_of(a.n);
    const int64_t groups = s.threads / (s.warps * 32), blocks = (a.rows + groups - 1) / groups;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_chain(GLR_BY_SHAPE(norm_kernel, T), dim3(static_cast<unsigned>(blocks)), s.threads, 0, st, a, s.warps,
                        reinterpret_cast<uintptr_t>(a.codes) % 8 == 0 && (a.rows == 1 || a.ld_codes % 8 == 0));
}
template <class T>
cudaError_t launch_grad(const NormGrad& a, int64_t blocks, cudaStream_t st) {
    const Shape s = shape_of(a.n);
    return launch_chain(GLR_BY_SHAPE(norm_grad_kernel, T), dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.nodes)), s.threads,
                        s.warps == 1 ? a.n * sizeof(float) : 0, st, a, s.warps);
}

}  // namespace

cudaError_t norm(const Norm& a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, several = a.rows > 1;
    const bool wide = a.n * es % 16 == 0 && on16(a.X, several * a.ldx * es) && on16(a.residual, several * a.ldr * es) &&
                      on16(a.H, several * a.ldh * es) && on16(a.Y, several * a.ldy * es) && on16(a.weight, 0);
    const int ctas = ring_ctas(a.n, 2, es);
    if (ctas > 0 && wide) {
        const int t = ring_threads(a.n);
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.rows, 152 * ctas)));
        return dtype == GLR_BF16 ? launch_ring(GLR_BY_THREADS(norm_ring_kernel, __nv_bfloat16, t), a, grid, t, ring_bytes(t, 2, es), st)
                                 : launch_ring(GLR_BY_THREADS(norm_ring_kernel, float, t), a, grid, t, ring_bytes(t, 2, es), st);
    }
    return dtype == GLR_BF16 ? launch_norm<__nv_bfloat16>(a, st) : launch_norm<float>(a, st);
}

// The partial sums' CTAs of either kernel (the ring kernels' are those of bf16 rows, of which an SM holds more).
int64_t ring_blocks(int64_t nodes, int64_t rows, int ctas) { return std::max<int64_t>(1, std::min<int64_t>(rows, 152 * ctas / nodes)); }
int64_t norm_grad_bytes(int64_t nodes, int64_t rows, int n) {
    const int ctas = ring_ctas(n, 3, 2);
    return nodes * std::max(grad_blocks(nodes, rows, n), ctas ? ring_blocks(nodes, rows, ctas) : 0) * n * 4;
}

cudaError_t norm_grad(const NormGrad& a, int dtype, int grad_dtype, cudaStream_t st) {
    if (a.rows == 0 && !a.want_dweight) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, several = a.nodes * a.rows > 1;
    const bool wide = a.n * es % 16 == 0 && on16(a.dX, several * a.lddx * es) && on16(a.residual, several * a.ldr * es) &&
                      on16(a.H, several * a.ldh * es) && on16(a.dY, several * a.lddy * es) && on16(a.weight, 0);
    const int ctas = ring_ctas(a.n, 3, es);
    int64_t blocks = grad_blocks(a.nodes, a.rows, a.n);
    cudaError_t e;
    if (ctas > 0 && wide) {
        const int t = ring_threads(a.n);
        blocks = ring_blocks(a.nodes, a.rows, ctas);
        const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(a.nodes));
        e = dtype == GLR_BF16 ? launch_ring(GLR_BY_THREADS(norm_grad_ring_kernel, __nv_bfloat16, t), a, grid, t, ring_bytes(t, 3, es), st)
                              : launch_ring(GLR_BY_THREADS(norm_grad_ring_kernel, float, t), a, grid, t, ring_bytes(t, 3, es), st);
    } else {
        e = dtype == GLR_BF16 ? launch_grad<__nv_bfloat16>(a, blocks, st) : launch_grad<float>(a, blocks, st);
    }
    if (e != cudaSuccess || !a.want_dweight) return e;
    const dim3 grid((a.n + 31) / 32, static_cast<unsigned>(a.nodes));
    return grad_dtype == GLR_BF16 ? launch_chain(norm_sum_kernel<__nv_bfloat16>, grid, kSumThreads, 0, st, a, static_cast<int>(blocks))
                                  : launch_chain(norm_sum_kernel<float>, grid, kSumThreads, 0, st, a, static_cast<int>(blocks));
}

}  // namespace rows
}  // namespace glr
