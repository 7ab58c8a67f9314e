// Arguments of the loss kernels (k_loss.cu), as the entry points (glr_operators.cu) fill them.
#pragma once

#include "glr_internal.cuh"

namespace glr {
namespace loss {

// An index array of int32 or int64; absent when p is null.
struct Index {
    const void* p;
    int wide;
    __device__ __forceinline__ int64_t at(int64_t i) const {
        return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
    }
};

// A row of the preference loss between its passes: its maximum, log2 of the sum of exp(z - maximum) (+infinity: the row does
// not count), and the factor of its gradient.
struct __align__(16) RowSum { float top, log2_sum, coef, unused; };

enum Kind : int { kDistill = 0, kPolicy = 1, kLogProb = 2 };

struct RowArgs {
    int64_t rows, vocab;
    const void* z; int64_t ldz;             // logits
    void* dz; int64_t lddz;                 // their gradient, or null
    const float* weight;                    // null: `share` each
    float share;
    float inv_tau;
    float* row_loss;
    // distillation
    const void* teacher; int64_t ldt; int teacher_bf16;
    Index ids; int64_t ldi; int topk;
    Index labels;
    float soft, hard;
    // policy
    Index tokens;                           // also the log-probability pass of the preference loss
    const float* old_logp; const float* advantage; const float* ref_logp;
    float clip_lo, clip_hi, kl;             // 1 - clip_low, 1 + clip_high
    float* logp;
    RowSum* sums;                           // log-probability pass: one a row
    int* err;
    int cluster_shift, slots, lists; uint32_t slot_bytes;    // set by the launcher
};

struct PairArgs {
    int64_t rows, pairs;
    Index offsets;
    const float* row_logp; RowSum* sums; const float* ref_logp; const float* weight;
    float share, beta, smoothing;
    int kind, average;
    float* pair_loss; float* seq_logp;
};

cudaError_t distill(const RowArgs& a, int dtype, cudaStream_t st);
cudaError_t policy(const RowArgs& a, int dtype, cudaStream_t st);
// row_logp (a.logp) and a.sums of every row, with coefficients of 0
cudaError_t log_prob(const RowArgs& a, int dtype, cudaStream_t st);
// pair losses, sequence sums, and sums[t].coef = d loss / d row_logp[t]
cudaError_t pairs(const PairArgs& a, cudaStream_t st);
// dz_t = coef (e_token - exp2((z - top) log2 e - log2_sum))
cudaError_t log_prob_grad(const RowArgs& a, int dtype, cudaStream_t st);
// *out = sum_t w_t x_t in a fixed order, w_t = weight[t] or share; entries of weight 0 add nothing
cudaError_t total(const float* x, const float* weight, float share, int64_t n, float* out, cudaStream_t st);

}  // namespace loss
}  // namespace glr
