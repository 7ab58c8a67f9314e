// Activations in 8 bits with a scale for every 32 columns, and back (the format is in glr_rows.cuh).  Four lanes hold a block,
// eight neighbouring columns each; a task of 32 threads is 512 columns of a row, two vectors a thread on their way at once.
// Bound by HBM (8192 x 5632 bf16 packed 25 us, unpacked 22, floor 21 each), unpacking with SiLU by its exponentials and
// reciprocals (30).
#include <algorithm>

#include "glr_linear.cuh"
#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kThreads = 256;

// Sixteen or 32 bytes of a row as they lie in memory; off 16 bytes element by element, each lane its own eight neighbours (8192 x 4095
// bf16 packed 41 us, 8192 x 4096 25, with the L2 flushed before).
template <class T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int n, bool wide) {
        if (wide && n >= 8) { u = *reinterpret_cast<const uint4*>(p); return; }
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = (2 * q < n ? h[2 * q] : 0u) | (2 * q + 1 < n ? h[2 * q + 1] : 0u) << 16;
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { widen8(u, v); }
    // the largest |x|, as an fp32 value's bits
    __device__ __forceinline__ uint32_t most() const {
        constexpr uint32_t m = 0x7fff7fffu;
        const uint32_t x = __vmaxu2(__vmaxu2(u.x & m, u.y & m), __vmaxu2(u.z & m, u.w & m));
        return max(x << 16, x & 0xffff0000u);
    }
};
template <> struct Raw<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* p, int n, bool wide) { load8(p, n, wide, v); }
    __device__ __forceinline__ void get(float (&to)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = v[e];
    }
    __device__ __forceinline__ uint32_t most() const {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
        return m;
    }
};

// Tasks of up to 32 threads (1 << shift), two vectors of eight columns each: `chunks` of a row, or two rows where a row has no more
// than one vector for each thread.
struct Tasks {
    int shift;
    int64_t chunks, all;
};
struct Pair {
    int64_t i[2], j[2];
    int n[2];
    __device__ __forceinline__ Pair(const Tasks& t, int64_t q, int64_t rows, int64_t cols) {
        const int64_t per8 = 8LL << t.shift, col = (threadIdx.x & ((1 << t.shift) - 1)) * 8;
        const bool one = cols <= per8;
        int64_t row = one ? 2 * q : q;
        if (t.chunks > 1) row = t.all <= 0x7fffffff ? static_cast<uint32_t>(q) / static_cast<uint32_t>(t.chunks) : q / t.chunks;
        i[0] = row; i[1] = one ? row + 1 : row;
        j[0] = one ? col : (q - row * t.chunks) * 2 * per8 + col;
        j[1] = one ? col : j[0] + per8;
#pragma unroll
        for (int u = 0; u < 2; ++u)
            n[u] = q < t.all && i[u] < rows ? static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(8), cols - j[u]))) : 0;
    }
};

template <class T>
__global__ void __launch_bounds__(kThreads) pack_kernel(const __grid_constant__ Pack a, const Tasks t, bool wide, bool wide_codes) {
    chain_begin();
    const int64_t group = kThreads >> t.shift;
    // all lanes of a block are there: the loop goes by the CTA's first task
    for (int64_t first = blockIdx.x * group; first < t.all; first += gridDim.x * group) {
        const Pair at(t, first + (threadIdx.x >> t.shift), a.rows, a.cols);
        Raw<T> x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) x[u].load(static_cast<const T*>(a.X) + at.i[u] * a.ldx + at.j[u], at.n[u], wide);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t m = x[u].most();
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const uint32_t s = scale_of(m);
            if (at.n[u] <= 0) continue;
            float v[8];
            x[u].get(v);
            store_codes(a.codes + at.i[u] * a.ld_codes + at.j[u], at.n[u], wide_codes, block_codes(v, s));
            if ((threadIdx.x & 3) == 0) a.scales[at.i[u] * a.ld_scales + at.j[u] / kBlock] = static_cast<uint8_t>(s);
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const __grid_constant__ Unpack a, const Tasks t) {
    chain_begin();
    const int64_t group = kThreads >> t.shift;
    for (int64_t first = blockIdx.x * group; first < t.all; first += gridDim.x * group) {
        const Pair at(t, first + (threadIdx.x >> t.shift), a.rows, a.cols);
        uint2 codes[2];
        uint32_t s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            codes[u] = load_codes(a.codes + at.i[u] * a.ld_codes + at.j[u], at.n[u], true);
            s[u] = at.n[u] > 0 ? a.scales[at.i[u] * a.ld_scales + at.j[u] / kBlock] : 0;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (at.n[u] <= 0) continue;
            float v[8];
            code_values(codes[u], s[u], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = linear::act_value<sizeof(T) == 2>(v[e], a.act);
            store8(static_cast<T*>(a.Y) + at.i[u] * a.ldy + at.j[u], at.n[u], true, v);
        }
    }
}

// The same of rows on 16 bytes (codes on 8) that are whole vectors, up to 2^31 tasks of a row each: both kernels are bound by
// what they issue (8192 x 5632 bf16 packed, with the index arithmetic above, 34 us at 0.8 of the issue slots).
struct Whole {
    int64_t row;
    uint32_t col;
    bool in[2];
    __device__ __forceinline__ Whole(const Tasks& t, uint32_t q, uint32_t cols) {
        const uint32_t r = t.chunks == 1 ? q : q / static_cast<uint32_t>(t.chunks);
        row = r;
        col = ((q - r * static_cast<uint32_t>(t.chunks)) << (t.shift + 1) | (threadIdx.x & ((1u << t.shift) - 1))) * 8;
        in[0] = q < static_cast<uint32_t>(t.all) && col < cols;
        in[1] = q < static_cast<uint32_t>(t.all) && col + (8u << t.shift) < cols;
    }
};
template <class T>
__global__ void __launch_bounds__(kThreads) pack_whole_kernel(const __grid_constant__ Pack a, const Tasks t) {
    chain_begin();
    const uint32_t group = kThreads >> t.shift, next = 8u << t.shift;
    for (uint32_t first = blockIdx.x * group; first < static_cast<uint32_t>(t.all); first += gridDim.x * group) {
        const Whole at(t, first + (threadIdx.x >> t.shift), static_cast<uint32_t>(a.cols));
        const T* x = static_cast<const T*>(a.X) + at.row * a.ldx + at.col;
        int8_t* codes = a.codes + at.row * a.ld_codes + at.col;
        uint8_t* scales = a.scales + at.row * a.ld_scales + at.col / kBlock;
        Raw<T> v[2];
        v[0].load(x, at.in[0] ? 8 : 0, true);
        v[1].load(x + next, at.in[1] ? 8 : 0, true);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t m = v[u].most();
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const uint32_t s = scale_of(m);
            float f[8];
            v[u].get(f);
            const uint2 c = block_codes(f, s);
            if (at.in[u]) {
                *reinterpret_cast<uint2*>(codes + u * next) = c;
                if ((threadIdx.x & 3) == 0) scales[u * next / kBlock] = static_cast<uint8_t>(s);
            }
        }
    }
}
template <class T, int ACT>
__global__ void __launch_bounds__(kThreads) unpack_whole_kernel(const __grid_constant__ Unpack a, const Tasks t) {
    chain_begin();
    const uint32_t group = kThreads >> t.shift, next = 8u << t.shift;
    for (uint32_t first = blockIdx.x * group; first < static_cast<uint32_t>(t.all); first += gridDim.x * group) {
        const Whole at(t, first + (threadIdx.x >> t.shift), static_cast<uint32_t>(a.cols));
        const int8_t* codes = a.codes + at.row * a.ld_codes + at.col;
        const uint8_t* scales = a.scales + at.row * a.ld_scales + at.col / kBlock;
        T* y = static_cast<T*>(a.Y) + at.row * a.ldy + at.col;
        uint2 c[2];
        uint32_t s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            c[u] = at.in[u] ? *reinterpret_cast<const uint2*>(codes + u * next) : make_uint2(0, 0);
            s[u] = at.in[u] ? scales[u * next / kBlock] : 0;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (!at.in[u]) continue;
            float v[8];
            code_values(c[u], s[u], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = linear::act_value<sizeof(T) == 2>(v[e], ACT);
            store8(y + u * next, 8, true, v);
        }
    }
}

// Rows off 16 bytes (codes off 8): 256 columns a warp.
template <class T>
__global__ void __launch_bounds__(kThreads) unpack_apart_kernel(const __grid_constant__ Unpack a, int64_t parts) {
    chain_begin();
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); q < a.rows * parts; q += warps) {
        const int64_t i = q / parts, first = (q - i * parts) * 256;
        float v[8];
        load_blocks(a.codes + i * a.ld_codes, a.scales + i * a.ld_scales, first, a.cols, v);
        if (a.act != GLR_ACT_NONE)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = linear::act_value<sizeof(T) == 2>(v[e], a.act);
        store_apart(static_cast<T*>(a.Y) + i * a.ldy, first, a.cols, v);
    }
}

bool on(const void* p, int64_t ld_bytes, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0 && ld_bytes % to == 0; }

Tasks tasks_of(int64_t rows, int64_t cols) {
    Tasks t{2, 1, 0};
    while (t.shift < 5 && (8LL << t.shift) < cols) ++t.shift;
    if (cols <= (8LL << t.shift)) { t.all = (rows + 1) / 2; return t; }
    t.chunks = (cols + (16LL << t.shift) - 1) / (16LL << t.shift);
    t.all = rows * t.chunks;
    return t;
}
unsigned blocks_of(const Tasks& t) {
    const int64_t group = kThreads >> t.shift;
    return static_cast<unsigned>(std::min<int64_t>((t.all + group - 1) / group, 152 * 32));
}
template <class T>
auto unpack_of(int act) {
    return act == GLR_ACT_RELU ? unpack_whole_kernel<T, GLR_ACT_RELU> : act == GLR_ACT_GELU ? unpack_whole_kernel<T, GLR_ACT_GELU>
         : act == GLR_ACT_GELU_TANH ? unpack_whole_kernel<T, GLR_ACT_GELU_TANH> : act == GLR_ACT_SILU ? unpack_whole_kernel<T, GLR_ACT_SILU>
                                    : unpack_whole_kernel<T, GLR_ACT_NONE>;
}
bool whole(const Tasks& t, int64_t cols) { return cols % 8 == 0 && cols > (8LL << t.shift) && t.all < (int64_t{1} << 31) - 152 * 32 * kThreads; }
unsigned apart_blocks(int64_t tasks) { return static_cast<unsigned>(std::min<int64_t>((tasks + kThreads / 32 - 1) / (kThreads / 32), 152 * 32)); }

}  // namespace

cudaError_t pack(const Pack& a, int dtype, cudaStream_t st) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4;
    const bool wide = on(a.X, a.rows > 1 ? a.ldx * es : 0, 16), wide_codes = on(a.codes, a.rows > 1 ? a.ld_codes : 0, 8);
    const Tasks t = tasks_of(a.rows, a.cols);
    const dim3 grid(blocks_of(t));
    if (wide && wide_codes && whole(t, a.cols))
        return dtype == GLR_BF16 ? launch_chain(pack_whole_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, t)
                                 : launch_chain(pack_whole_kernel<float>, grid, kThreads, 0, st, a, t);
    return dtype == GLR_BF16 ? launch_chain(pack_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, t, wide, wide_codes)
                             : launch_chain(pack_kernel<float>, grid, kThreads, 0, st, a, t, wide, wide_codes);
}

cudaError_t unpack(const Unpack& a, int dtype, cudaStream_t st) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, several = a.rows > 1;
    if (!on(a.Y, several * a.ldy * es, 16) || !on(a.codes, several * a.ld_codes, 8)) {
        const int64_t parts = (a.cols + 255) / 256;
        return dtype == GLR_BF16 ? launch_chain(unpack_apart_kernel<__nv_bfloat16>, apart_blocks(a.rows * parts), kThreads, 0, st, a, parts)
                                 : launch_chain(unpack_apart_kernel<float>, apart_blocks(a.rows * parts), kThreads, 0, st, a, parts);
    }
    const Tasks t = tasks_of(a.rows, a.cols);
    const dim3 grid(blocks_of(t));
    if (whole(t, a.cols))
        return dtype == GLR_BF16 ? launch_chain(unpack_of<__nv_bfloat16>(a.act), grid, kThreads, 0, st, a, t)
                                 : launch_chain(unpack_of<float>(a.act), grid, kThreads, 0, st, a, t);
    return dtype == GLR_BF16 ? launch_chain(unpack_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, t)
                             : launch_chain(unpack_kernel<float>, grid, kThreads, 0, st, a, t);
}

}  // namespace rows
}  // namespace glr
