// Arguments of the row kernels (embeddings, norms, 8-bit checkpoints, token log-probabilities), as the entry points
// (glr_rows.cu) fill them, and the loads and stores they share.
#pragma once

#include "glr_internal.cuh"

namespace glr {
namespace rows {

// An index array of int32 or int64; absent when p is null.
struct Index {
    const void* p;
    int wide;
    __device__ __forceinline__ int64_t at(int64_t i) const {
        return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
    }
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ void widen8(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[2 * q] = __uint_as_float(w[q] << 16); v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u); }
}
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Eight neighbouring elements of a row, `n` of them there (the others are 0): in 16-byte loads where `wide` says that rows
// lie so, one by one else.  (Plain loads: ones through the path for constant data may be moved before chain_begin.)
template <class T>
__device__ __forceinline__ void load8(const T* p, int n, bool wide, float (&v)[8]) {
    if (wide && n >= 8) {
        if (sizeof(T) == 2) {
            widen8(*reinterpret_cast<const uint4*>(p), v);
        } else {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f(p[e]) : 0.f;
    }
}
template <class T>
__device__ __forceinline__ void store8(T* p, int n, bool wide, const float (&v)[8]) {
    if (wide && n >= 8) {
        if (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(p) = make_uint4(narrow2(v[0], v[1]), narrow2(v[2], v[3]), narrow2(v[4], v[5]), narrow2(v[6], v[7]));
        } else {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) put(p + e, v[e]);
    }
}

// Where rows do not lie on 16 bytes, a warp takes 256 columns with each lane's eight 32 apart, so that neighbouring lanes
// touch neighbouring elements (each lane's eight next to each other cost four times the L1's cycles: a norm of 8192 x 4095 bf16
// 87 us instead of 49, its gradient 227 instead of 109).
template <class T>
__device__ __forceinline__ void load_apart(const T* row, int64_t first, int64_t cols, float (&v)[8]) {
    const int64_t j = first + (threadIdx.x & 31);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = j + e * 32 < cols ? to_f(row[j + e * 32]) : 0.f;
}
template <class T>
__device__ __forceinline__ void store_apart(T* row, int64_t first, int64_t cols, const float (&v)[8]) {
    const int64_t j = first + (threadIdx.x & 31);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e * 32 < cols) put(row + j + e * 32, v[e]);
}

// ---- blocks of 32 columns in 8 bits ----------------------------------------------------------------------------
// A block's scale is the smallest power of two s with amax <= 127 s, at least 2^-127 and at most 2^121, stored as its exponent
// plus 127; a code is x / s rounded to the nearest integer, ties to even, and at most 127 (which 2^121, whose double would
// have 2^128 among its values, needs for |x| above 127.5 2^121).  x / s is exact, so the codes are the same whoever makes
// them, and code * s is exact in bf16 and fp32.  A block with an infinity or a NaN has the scale 255 and stands for NaN.
constexpr int kBlock = 32;
constexpr uint32_t kNoScale = 255, kTopScale = 248;

// ... from the largest |x| of the block as an integer (its order is that of the values, NaN above all).
__device__ __forceinline__ uint32_t scale_of(uint32_t amax) {
    const uint32_t e = amax >> 23;
    if (e == 255) return kNoScale;
    const uint32_t up = e + ((amax & 0x7fffffu) > 0x7e0000u ? 1u : 0u);      // mantissa above 127 / 64
    return up > 6 ? min(up - 6, kTopScale) : 0;
}
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }     // s <= 248
__device__ __forceinline__ float scale_value(uint32_t s) {
    return s == kNoScale ? __uint_as_float(0x7fffffffu) : __uint_as_float(s ? s << 23 : 0x00400000u);
}
// Four neighbouring lanes hold a block, eight elements each.
__device__ __forceinline__ uint32_t block_scale(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    return scale_of(m);
}
// The nearest integer to a product of at most 127 stands in the low bits of its sum with 1.5 2^23.
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, uint32_t scale) {
    if (scale == kNoScale) return 0;
    const float inv = inverse_scale(scale), half = 12582912.f;
    int q[4] = {__float_as_int(fmaf(a, inv, half)), __float_as_int(fmaf(b, inv, half)), __float_as_int(fmaf(c, inv, half)),
                __float_as_int(fmaf(d, inv, half))};
    if (scale == kTopScale) {
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = max(0x4b400000 - 127, min(0x4b400000 + 127, q[e]));
    }
    return __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
}
__device__ __forceinline__ uint2 block_codes(const float (&v)[8], uint32_t scale) {
    return make_uint2(four_codes(v[0], v[1], v[2], v[3], scale), four_codes(v[4], v[5], v[6], v[7], scale));
}
__device__ __forceinline__ void code_values(uint2 c, uint32_t scale, float (&v)[8]) {
    const float s = scale_value(scale);
    const uint32_t w[2] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u};        // codes + 128, each the low byte of 2^23 + code + 128
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__uint_as_float(__byte_perm(w[e / 4], 0x4b000000u, 0x7650 + e % 4)) - 8388736.f) * s;
}
__device__ __forceinline__ void store_codes(int8_t* p, int n, bool wide, uint2 c) {
    if (wide && n >= 8) {
        *reinterpret_cast<uint2*>(p) = c;
    } else {
        const uint32_t w[2] = {c.x, c.y};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = static_cast<int8_t>(w[e / 4] >> (8 * (e % 4)));
    }
}
__device__ __forceinline__ uint2 load_codes(const int8_t* p, int n, bool wide) {
    if (wide && n >= 8) return *reinterpret_cast<const uint2*>(p);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) w[e / 4] |= static_cast<uint32_t>(static_cast<uint8_t>(p[e])) << (8 * (e % 4));
    return make_uint2(w[0], w[1]);
}

// 256 columns that the lanes hold apart, in 8 bits: turned round in `turn` (256 floats, the warp's own) first.
__device__ __forceinline__ void store_blocks(int8_t* codes, uint8_t* scales, int64_t first, int64_t cols, bool wide, float (&v)[8], float* turn) {
    const int lane = threadIdx.x & 31;
    const int64_t j = first + lane * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) turn[e * 32 + lane] = v[e];
    __syncwarp();
    const float4 a = reinterpret_cast<const float4*>(turn)[2 * lane], b = reinterpret_cast<const float4*>(turn)[2 * lane + 1];
    __syncwarp();
    const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const uint32_t s = block_scale(w);
    const uint2 c = block_codes(w, s);
    if (j < cols) {
        store_codes(codes + j, static_cast<int>(min(static_cast<int64_t>(8), cols - j)), wide, c);
        if ((lane & 3) == 0) scales[j / kBlock] = static_cast<uint8_t>(s);
    }
}
__device__ __forceinline__ void load_blocks(const int8_t* codes, const uint8_t* scales, int64_t first, int64_t cols, float (&v)[8]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t j = first + e * 32;
        v[e] = j + lane < cols ? static_cast<float>(codes[j + lane]) * scale_value(scales[j / kBlock]) : 0.f;
    }
}

// ---- arguments ---------------------------------------------------------------------------------------------------
struct Lookup {
    int64_t rows, vocab, d;
    const void* E; int64_t lde;
    Index tokens;
    void* Y; int64_t ldy;
    float scale;
};
cudaError_t lookup(const Lookup& a, int dtype, cudaStream_t st);

struct EmbeddingGrad {
    int64_t nodes, rows, vocab, d;
    const void* dY; int64_t lddy;
    Index tokens;
    float scale;
    int accumulate;
    void* dE[GLR_MAX_NODES];
    void* workspace;
};
int64_t embedding_grad_bytes(int64_t nodes, int64_t rows, int64_t vocab, int64_t d);
cudaError_t embedding_grad(const EmbeddingGrad& a, int dtype, int grad_dtype, cudaStream_t st);

constexpr int kMaxNorm = GLR_MAX_NORM;
struct Norm {
    int64_t rows; int n;
    const void* X; int64_t ldx;
    const void* residual; int64_t ldr;
    const void* weight;
    void* H; int64_t ldh;
    void* Y; int64_t ldy;
    float* rstd;
    int8_t* codes; int64_t ld_codes;
    uint8_t* scales; int64_t ld_scales;
    float eps;
};
cudaError_t norm(const Norm& a, int dtype, cudaStream_t st);

struct NormGrad {
    int64_t nodes, rows; int n;
    const void* dY; int64_t lddy;
    const void* H; int64_t ldh;
    const float* rstd;
    const void* weight;
    const void* residual; int64_t ldr;
    void* dX; int64_t lddx;
    void* dweight[GLR_MAX_NODES];
    int want_dweight;
    float* partial;                          // norm_grad_bytes
};
int64_t norm_grad_bytes(int64_t nodes, int64_t rows, int n);
cudaError_t norm_grad(const NormGrad& a, int dtype, int grad_dtype, cudaStream_t st);

struct Pack {
    int64_t rows, cols;
    const void* X; int64_t ldx;
    int8_t* codes; int64_t ld_codes;
    uint8_t* scales; int64_t ld_scales;
};
cudaError_t pack(const Pack& a, int dtype, cudaStream_t st);
// Y receives act(value).
struct Unpack {
    int64_t rows, cols;
    const int8_t* codes; int64_t ld_codes;
    const uint8_t* scales; int64_t ld_scales;
    void* Y; int64_t ldy;
    int act;
};
cudaError_t unpack(const Unpack& a, int dtype, cudaStream_t st);

struct TokenLogp {
    int64_t rows, vocab; int topk;
    const void* z; int64_t ldz;
    Index tokens;
    float* logp; float* lse; float* entropy;
    float* top_logp; int64_t ld_top_logp;
    void* top_ids; int64_t ld_top_ids; int ids_wide;
    float inv_tau;
};
cudaError_t token_logp(const TokenLogp& a, int dtype, cudaStream_t st);

struct TokenLogpGrad {
    int64_t rows, vocab;
    const void* z; int64_t ldz;
    Index tokens;
    const float* lse; const float* entropy; const float* dlogp; const float* dentropy;
    void* dz; int64_t lddz;
    float inv_tau;
};
cudaError_t token_logp_grad(const TokenLogpGrad& a, int dtype, cudaStream_t st);

}  // namespace rows
}  // namespace glr
