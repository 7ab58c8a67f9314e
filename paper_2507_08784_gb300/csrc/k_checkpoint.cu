// Activations in 8 bits with a scale for every 32 columns, and back (the format is in glr_rows.cuh): bound by HBM.  A row
// has 4 to 256 threads (a power of two) with eight neighbouring elements each, so that four lanes hold a block.
#include <algorithm>

#include "glr_linear.cuh"
#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kThreads = 256;

template <class T>
__global__ void __launch_bounds__(kThreads) pack_kernel(const __grid_constant__ Pack a, int shift, bool wide, bool wide_codes) {
    chain_begin();
    const int per = 1 << shift, at = threadIdx.x & (per - 1);
    const int64_t up = (a.cols + kBlock - 1) / kBlock * kBlock, step = static_cast<int64_t>(gridDim.x) * (kThreads >> shift);
    // a warp's lanes may hold several rows: all of them stay until the last one's row is done
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads >> shift); first < a.rows; first += step) {
        const int64_t i = first + (threadIdx.x >> shift);
        const bool here = i < a.rows;
        const T* x = static_cast<const T*>(a.X) + (here ? i : 0) * a.ldx;
        for (int64_t j = at * 8; j - at * 8 < up; j += per * 8) {
            const int n = here ? static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(8), a.cols - j))) : 0;
            float v[8];
            load8(x + j, n, wide, v);
            const uint32_t s = block_scale(v);
            const uint2 c = block_codes(v, s);
            if (n > 0) {
                store_codes(a.codes + i * a.ld_codes + j, n, wide_codes, c);
                if ((at & 3) == 0) a.scales[i * a.ld_scales + j / kBlock] = static_cast<uint8_t>(s);
            }
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const __grid_constant__ Unpack a, int shift) {
    chain_begin();
    const int per = 1 << shift;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads >> shift);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kThreads >> shift) + (threadIdx.x >> shift); i < a.rows; i += step)
        for (int64_t j = (threadIdx.x & (per - 1)) * 8; j < a.cols; j += per * 8) {
            const int n = static_cast<int>(min(static_cast<int64_t>(8), a.cols - j));
            float v[8];
            code_values(load_codes(a.codes + i * a.ld_codes + j, n, true), a.scales[i * a.ld_scales + j / kBlock], v);
            if (a.Z) store8(static_cast<T*>(a.Z) + i * a.ldz + j, n, true, v);
            if (!a.Y) continue;
            if (a.act != GLR_ACT_NONE)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = linear::act_value<sizeof(T) == 2>(v[e], a.act);
            store8(static_cast<T*>(a.Y) + i * a.ldy + j, n, true, v);
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
        if (a.Z) store_apart(static_cast<T*>(a.Z) + i * a.ldz, first, a.cols, v);
        if (!a.Y) continue;
        if (a.act != GLR_ACT_NONE)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = linear::act_value<sizeof(T) == 2>(v[e], a.act);
        store_apart(static_cast<T*>(a.Y) + i * a.ldy, first, a.cols, v);
    }
}

bool on(const void* p, int64_t ld_bytes, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0 && ld_bytes % to == 0; }

int threads_shift(int64_t cols) {
    int shift = 2;
    while (shift < 8 && (8LL << shift) < cols) ++shift;
    return shift;
}
unsigned blocks_of(int64_t rows, int shift) {
    return static_cast<unsigned>(std::min<int64_t>((rows + (kThreads >> shift) - 1) / (kThreads >> shift), 152 * 32));
}

unsigned apart_blocks(int64_t tasks) { return static_cast<unsigned>(std::min<int64_t>((tasks + kThreads / 32 - 1) / (kThreads / 32), 152 * 32)); }

}  // namespace

cudaError_t pack(const Pack& a, int dtype, cudaStream_t st) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4;
    const bool wide = on(a.X, a.rows > 1 ? a.ldx * es : 0, 16), wide_codes = on(a.codes, a.rows > 1 ? a.ld_codes : 0, 8);
    const int shift = threads_shift(a.cols);
    const dim3 grid(blocks_of(a.rows, shift));
    return dtype == GLR_BF16 ? launch_chain(pack_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, shift, wide, wide_codes)
                             : launch_chain(pack_kernel<float>, grid, kThreads, 0, st, a, shift, wide, wide_codes);
}

cudaError_t unpack(const Unpack& a, int dtype, cudaStream_t st) {
    if (a.rows == 0 || a.cols == 0 || (!a.Y && !a.Z)) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, several = a.rows > 1;
    if ((a.Y && !on(a.Y, several * a.ldy * es, 16)) || (a.Z && !on(a.Z, several * a.ldz * es, 16)) || !on(a.codes, several * a.ld_codes, 8)) {
        const int64_t parts = (a.cols + 255) / 256;
        return dtype == GLR_BF16 ? launch_chain(unpack_apart_kernel<__nv_bfloat16>, apart_blocks(a.rows * parts), kThreads, 0, st, a, parts)
                                 : launch_chain(unpack_apart_kernel<float>, apart_blocks(a.rows * parts), kThreads, 0, st, a, parts);
    }
    const int shift = threads_shift(a.cols);
    const dim3 grid(blocks_of(a.rows, shift));
    return dtype == GLR_BF16 ? launch_chain(unpack_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a, shift)
                             : launch_chain(unpack_kernel<float>, grid, kThreads, 0, st, a, shift);
}

}  // namespace rows
}  // namespace glr
