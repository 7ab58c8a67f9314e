// Arguments of the linear layers' kernels, as the entry points (glr_operators.cu) fill them.
#pragma once

#include "glr_internal.cuh"

namespace glr {
namespace linear {

// What the epilogue makes of an element acc of the product:
//   kForward    z = acc + bias; aux <- z; out <- act(z) + add
//   kGradInput  g = acc + add; aux <- g; out <- g act'(pre)
//   kGradWeight out[node] <- acc
enum Mode : int { kForward = 0, kGradInput = 1, kGradWeight = 2 };

// out(i, j) = epilogue(sum_p A(i, p) B(j, p)), i < M, j < N, p < K, for every node (batch) b: A and B
// move on by sAb and sBb elements.  A(i, p) = A[i sAi + p sAp], one of sAi and sAp being 1; B alike.
struct Product {
    int mode, dtype, out_dtype, act;
    int64_t M, N, K;
    int nodes;
    const void* A; int64_t sAi, sAp, sAb;
    const void* B; int64_t sBj, sBp, sBb;
    void* out; int64_t ldo;
    const void* bias;
    const void* add; int64_t ldadd;
    const void* pre; int64_t ldpre;
    void* aux; int64_t ldaux;
    void* outs[GLR_MAX_NODES];              // kGradWeight: each node's M x N result, contiguous
    int* err;
};

// tcgen05 (k_linear_tc.cu): whether it takes the product, and the workspace that the packed operands need.
struct TcPlan {
    bool ok, pack_a, pack_b;
    int planes;
    int64_t bytes_a, bytes_b;
    int64_t bytes() const { return ok ? bytes_a + bytes_b : 0; }
};
TcPlan tc_plan(const Product& p);
cudaError_t tc_product(const Product& p, const TcPlan& plan, void* workspace, cudaStream_t st);
// Any strides, sizes, alignment and types, without workspace (k_linear.cu).
cudaError_t any_product(const Product& p, cudaStream_t st);
double any_cost(const Product& p);              // its time, us (measured fit)
// Which kernels a product's sizes and alignment call for; without the workspace that `tc` asks for, kAny.
enum class Way { kNone, kFewRows, kTensorCores, kAny };
struct Plan { Way way; TcPlan tc; };
Plan plan_of(const Product& p);
cudaError_t product(const Product& p, void* workspace, int64_t workspace_bytes, cudaStream_t st);
int sm_count();                                 // of the current device; 152 without one

// sums[b][j] = sum over the rows of node b of x(i, j), x rows x n in rows of ldx
struct ColumnSums {
    int64_t rows, n;
    int nodes, dtype, out_dtype;
    const void* x; int64_t ldx;
    void* sums[GLR_MAX_NODES];
};
cudaError_t column_sums(const ColumnSums& c, cudaStream_t st);

// The activations and their slopes (GLR_ACT_*).  FAST, for results that are rounded to bf16: exponentials and
// quotients by the hardware's approximations (a few 2^-22 relative, an exponential's more with its argument), tanh u as
// 1 - 2 / (1 + exp(2 u)).
template <bool FAST>
__device__ __forceinline__ float exp_of(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST>
__device__ __forceinline__ float tanh_of(float u) {
    // (beyond 40 the quotient's denominator would leave the range of the fast division)
    return FAST ? 1.f - __fdividef(2.f, 1.f + __expf(2.f * fminf(u, 40.f))) : tanhf(u);
}
template <bool FAST>
__device__ __forceinline__ float sigmoid_of(float z) {
    if (!FAST) return 1.f / (1.f + expf(-z));
    // from exp(-|z|): nothing leaves the fast division's range, and the value goes to 0 where exp(z) does
    const float e = __expf(-fabsf(z));
    return __fdividef(z >= 0.f ? 1.f : e, 1.f + e);
}
template <bool FAST>
__device__ __forceinline__ float act_value(float z, int act) {
    switch (act) {
        case GLR_ACT_RELU: return z <= 0.f ? 0.f : z;            // a NaN stays one
        case GLR_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.7071067811865476f));
        case GLR_ACT_GELU_TANH: return 0.5f * z * (1.f + tanh_of<FAST>(0.7978845608028654f * (z + 0.044715f * z * z * z)));
        case GLR_ACT_SILU: return FAST ? z * sigmoid_of<FAST>(z) : z / (1.f + expf(-z));
        default: return z;
    }
}
template <bool FAST>
__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
        case GLR_ACT_RELU: return z <= 0.f ? 0.f : z > 0.f ? 1.f : z;
        case GLR_ACT_GELU:
            return 0.5f * (1.f + erff(z * 0.7071067811865476f)) + z * (0.3989422804014327f * exp_of<FAST>(-0.5f * z * z));
        case GLR_ACT_GELU_TANH: {
            const float t = tanh_of<FAST>(0.7978845608028654f * (z + 0.044715f * z * z * z));
            const float z2 = fminf(z * z, 1e9f);       // (1 - t t is 0 long before)
            return 0.5f * (1.f + t) + 0.5f * z * (1.f - t * t) * 0.7978845608028654f * (1.f + 3.f * 0.044715f * z2);
        }
        case GLR_ACT_SILU: {
            const float p = sigmoid_of<FAST>(z);
            return p * (1.f + z * (1.f - p));
        }
        default: return 1.f;
    }
}

}  // namespace linear
}  // namespace glr
