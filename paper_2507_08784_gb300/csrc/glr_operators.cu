// Entry points of the operators around the step: linear layers and the losses on logits.  They check their arguments, fill
// the kernels' arguments and launch; nothing is kept between calls and nothing is allocated.
#include <cstdarg>
#include <cstdio>
#include <mutex>

#include "glr_linear.cuh"
#include "glr_loss.cuh"

namespace glr {
namespace {

int refuse(const char* fmt, ...) {
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    set_global_error(msg);
    return GLR_EINVAL;
}
int launched(const char* who, cudaError_t e) {
    if (e == cudaSuccess) return GLR_OK;
    char msg[256];
    snprintf(msg, sizeof(msg), "%s: launch failed: %s", who, cudaGetErrorString(e));
    set_global_error(msg);
    return GLR_ECUDA;
}

// Bounded waits that gave up, per device (glr_operator_status).
__device__ int g_gave_up;
constexpr int kMaxDevices = 256;
std::mutex g_mutex;
int* g_gave_up_addr[kMaxDevices] = {};

int* gave_up_counter() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!g_gave_up_addr[dev]) {
        void* p = nullptr;
        if (cudaGetSymbolAddress(&p, g_gave_up) != cudaSuccess) { cudaGetLastError(); return nullptr; }
        g_gave_up_addr[dev] = static_cast<int*>(p);
    }
    return g_gave_up_addr[dev];
}

inline int64_t bytes_of(int dtype) { return dtype == GLR_BF16 ? 2 : 4; }
inline bool dtype_ok(int dtype) { return dtype == GLR_F32 || dtype == GLR_BF16; }

// A row-major matrix argument: present where it has elements, rows no closer than their length,
// elements on their own size.
bool matrix_ok(const void* p, int64_t ld, int64_t rows, int64_t cols, int dtype) {
    if (rows == 0 || cols == 0) return true;
    return p && (rows == 1 || ld >= cols) && reinterpret_cast<uintptr_t>(p) % bytes_of(dtype) == 0;
}
bool vector_ok(const void* p, int64_t n, int64_t bytes) {
    return n == 0 || (p && reinterpret_cast<uintptr_t>(p) % bytes == 0);
}
bool optional_ok(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

constexpr int64_t kMaxRows = int64_t(1) << 24;

// The checks all losses share.
int check_logits(const char* who, int64_t rows, int64_t vocab, const void* z, int64_t ldz, void* dz, int64_t lddz,
                 const float* weight, float* loss, int dtype) {
    if (!dtype_ok(dtype)) return refuse("%s: unknown dtype %d", who, dtype);
    if (rows < 0 || rows > kMaxRows) return refuse("%s: need 0 <= rows <= 2^24", who);
    if (vocab < 1 || vocab > GLR_MAX_LOGIT_BYTES || vocab * bytes_of(dtype) > GLR_MAX_LOGIT_BYTES)
        return refuse("%s: need vocab >= 1 and rows of logits of at most %d bytes", who, GLR_MAX_LOGIT_BYTES);
    if (!matrix_ok(z, ldz, rows, vocab, dtype)) return refuse("%s: logits null, misaligned or with ld < vocab", who);
    if (dz && !matrix_ok(dz, lddz, rows, vocab, dtype)) return refuse("%s: dlogits misaligned or with ld < vocab", who);
    if (dz && dz == z && rows > 1 && ldz != lddz) return refuse("%s: dlogits in place of logits needs the same ld", who);
    if (!optional_ok(weight, 4)) return refuse("%s: weight misaligned", who);
    if (!vector_ok(loss, 1, 4)) return refuse("%s: loss is null or misaligned", who);
    return GLR_OK;
}
// ... and those of the linear layers: the products' tiles are counted in 32 bits.
int check_layer(const char* who, int64_t rows, int64_t n, int64_t k, int dtype, int act) {
    if (!dtype_ok(dtype)) return refuse("%s: unknown dtype %d", who, dtype);
    if (act < GLR_ACT_NONE || act > GLR_ACT_SILU) return refuse("%s: unknown activation %d", who, act);
    if (rows < 0 || n < 0 || k < 0 || rows > (int64_t(1) << 30) || n > (int64_t(1) << 24) || k > (int64_t(1) << 24))
        return refuse("%s: need 0 <= rows <= 2^30 and 0 <= n, k <= 2^24", who);
    return GLR_OK;
}
bool positive(float x) { return x >= 1.2e-38f && x <= 3.0e38f; }       // its reciprocal too
bool finite(float x) { return x >= -3.0e38f && x <= 3.0e38f; }
bool flag(int v) { return v == 0 || v == 1; }

}  // namespace
}  // namespace glr

using namespace glr;

namespace {

// The checks and the product of a call.
int linear_product(const char* who, const glr_linear_args* a, linear::Product& p) {
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_layer(who, a->rows, a->n, a->k, a->dtype, a->act)) return rc;
    if (!matrix_ok(a->X, a->ldx, a->rows, a->k, a->dtype) || !matrix_ok(a->W, a->ldw, a->n, a->k, a->dtype))
        return refuse("%s: X or W null, misaligned or with ld < k", who);
    if (!matrix_ok(a->Y, a->ldy, a->rows, a->n, a->dtype)) return refuse("%s: Y null, misaligned or with ld < n", who);
    if (!optional_ok(a->bias, bytes_of(a->dtype))) return refuse("%s: bias misaligned", who);
    if (a->residual && !matrix_ok(a->residual, a->ldr, a->rows, a->n, a->dtype))
        return refuse("%s: residual misaligned or with ld < n", who);
    if (a->preact && !matrix_ok(a->preact, a->ldp, a->rows, a->n, a->dtype))
        return refuse("%s: preact misaligned or with ld < n", who);
    if (a->residual && a->residual == a->Y && a->rows > 1 && a->ldr != a->ldy)
        return refuse("%s: residual in place of Y needs the same ld", who);
    p = linear::Product{};
    p.mode = linear::kForward; p.dtype = p.out_dtype = a->dtype; p.act = a->act;
    p.M = a->rows; p.N = a->n; p.K = a->k; p.nodes = 1;
    p.A = a->X; p.sAi = a->ldx; p.sAp = 1;
    p.B = a->W; p.sBj = a->ldw; p.sBp = 1;
    p.out = a->Y; p.ldo = a->ldy; p.bias = a->bias;
    p.add = a->residual; p.ldadd = a->ldr; p.aux = a->preact; p.ldaux = a->ldp;
    return GLR_OK;
}

int grad_input_product(const char* who, const glr_linear_grad_input_args* a, linear::Product& p) {
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_layer(who, a->rows, a->n, a->k, a->dtype, a->act)) return rc;
    if (!matrix_ok(a->dZ, a->lddz, a->rows, a->n, a->dtype)) return refuse("%s: dZ null, misaligned or with ld < n", who);
    if (!matrix_ok(a->W, a->ldw, a->n, a->k, a->dtype)) return refuse("%s: W null, misaligned or with ld < k", who);
    if (!matrix_ok(a->dX, a->lddx, a->rows, a->k, a->dtype)) return refuse("%s: dX null, misaligned or with ld < k", who);
    if (a->act != GLR_ACT_NONE && !a->preact && a->rows && a->k) return refuse("%s: an activation needs preact", who);
    if ((a->residual && !matrix_ok(a->residual, a->ldr, a->rows, a->k, a->dtype)) ||
        (a->preact && !matrix_ok(a->preact, a->ldp, a->rows, a->k, a->dtype)) ||
        (a->grad_out && !matrix_ok(a->grad_out, a->ldg, a->rows, a->k, a->dtype)))
        return refuse("%s: residual, preact or grad_out misaligned or with ld < k", who);
    if (a->residual && a->rows > 1 &&
        ((a->residual == a->dX && a->ldr != a->lddx) || (a->residual == a->grad_out && a->ldr != a->ldg)))
        return refuse("%s: residual in place of an output needs the same ld", who);
    p = linear::Product{};
    p.mode = linear::kGradInput; p.dtype = p.out_dtype = a->dtype; p.act = a->act;
    p.M = a->rows; p.N = a->k; p.K = a->n; p.nodes = 1;
    p.A = a->dZ; p.sAi = a->lddz; p.sAp = 1;
    p.B = a->W; p.sBj = 1; p.sBp = a->ldw;
    p.out = a->dX; p.ldo = a->lddx;
    p.add = a->residual; p.ldadd = a->ldr;
    if (a->act != GLR_ACT_NONE) { p.pre = a->preact; p.ldpre = a->ldp; }
    p.aux = a->grad_out; p.ldaux = a->ldg;
    return GLR_OK;
}

int grad_weight_product(const char* who, const glr_linear_grad_weight_args* a, linear::Product& p) {
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_layer(who, a->rows, a->n, a->k, a->dtype, GLR_ACT_NONE)) return rc;
    if (!dtype_ok(a->grad_dtype)) return refuse("%s: unknown grad_dtype %d", who, a->grad_dtype);
    if (a->nodes < 1 || a->nodes > GLR_MAX_NODES) return refuse("%s: need 1 <= nodes <= %d", who, GLR_MAX_NODES);
    const int64_t all = a->nodes * a->rows;
    if (!matrix_ok(a->dZ, a->lddz, all, a->n, a->dtype)) return refuse("%s: dZ null, misaligned or with ld < n", who);
    if (!matrix_ok(a->X, a->ldx, all, a->k, a->dtype)) return refuse("%s: X null, misaligned or with ld < k", who);
    if (!a->dW) return refuse("%s: dW is null", who);
    const int64_t gs = bytes_of(a->grad_dtype);
    for (int64_t i = 0; i < a->nodes; ++i) {
        if (!vector_ok(a->dW[i], a->n * a->k, gs)) return refuse("%s: dW[%d] is null or misaligned", who, (int)i);
        if (a->db && !vector_ok(a->db[i], a->n, gs)) return refuse("%s: db[%d] is null or misaligned", who, (int)i);
    }
    p = linear::Product{};
    p.mode = linear::kGradWeight; p.dtype = a->dtype; p.out_dtype = a->grad_dtype;
    p.M = a->n; p.N = a->k; p.K = a->rows; p.nodes = static_cast<int>(a->nodes);
    p.A = a->dZ; p.sAi = 1; p.sAp = a->lddz; p.sAb = a->rows * a->lddz;
    p.B = a->X; p.sBj = 1; p.sBp = a->ldx; p.sBb = a->rows * a->ldx;
    for (int64_t i = 0; i < a->nodes; ++i) p.outs[i] = a->dW[i];
    return GLR_OK;
}

int run_product(const char* who, linear::Product& p, void* workspace, int64_t bytes, cudaStream_t st) {
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return refuse("%s: workspace is not 16-byte aligned", who);
    if (!(p.err = gave_up_counter())) return launched(who, cudaErrorNoDevice);
    return launched(who, linear::product(p, workspace, bytes, st));
}
int product_workspace(int rc, const linear::Product& p, int64_t* bytes) {
    if (rc == GLR_OK) *bytes = linear::plan_of(p).tc.bytes();
    return rc;
}

}  // namespace

extern "C" int glr_linear(const glr_linear_args* a, void* stream) {
    linear::Product p;
    const int rc = linear_product("glr_linear", a, p);
    return rc ? rc : run_product("glr_linear", p, a->workspace, a->workspace_bytes, static_cast<cudaStream_t>(stream));
}
extern "C" int glr_linear_workspace(const glr_linear_args* a, int64_t* bytes) {
    linear::Product p;
    if (!bytes) return refuse("%s: bytes is null", "glr_linear_workspace");
    return product_workspace(linear_product("glr_linear_workspace", a, p), p, bytes);
}

extern "C" int glr_linear_grad_input(const glr_linear_grad_input_args* a, void* stream) {
    linear::Product p;
    const int rc = grad_input_product("glr_linear_grad_input", a, p);
    return rc ? rc : run_product("glr_linear_grad_input", p, a->workspace, a->workspace_bytes, static_cast<cudaStream_t>(stream));
}
extern "C" int glr_linear_grad_input_workspace(const glr_linear_grad_input_args* a, int64_t* bytes) {
    linear::Product p;
    if (!bytes) return refuse("%s: bytes is null", "glr_linear_grad_input_workspace");
    return product_workspace(grad_input_product("glr_linear_grad_input_workspace", a, p), p, bytes);
}

extern "C" int glr_linear_grad_weight(const glr_linear_grad_weight_args* a, void* stream) {
    const char* who = "glr_linear_grad_weight";
    linear::Product p;
    if (int rc = grad_weight_product(who, a, p)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (int rc = run_product(who, p, a->workspace, a->workspace_bytes, st)) return rc;
    if (!a->db) return GLR_OK;
    linear::ColumnSums c{};
    c.rows = a->rows; c.n = a->n; c.nodes = p.nodes; c.dtype = a->dtype; c.out_dtype = a->grad_dtype;
    c.x = a->dZ; c.ldx = a->lddz;
    for (int64_t i = 0; i < a->nodes; ++i) c.sums[i] = a->db[i];
    return launched(who, linear::column_sums(c, st));
}
extern "C" int glr_linear_grad_weight_workspace(const glr_linear_grad_weight_args* a, int64_t* bytes) {
    linear::Product p;
    if (!bytes) return refuse("%s: bytes is null", "glr_linear_grad_weight_workspace");
    return product_workspace(grad_weight_product("glr_linear_grad_weight_workspace", a, p), p, bytes);
}

extern "C" int glr_distill_loss(const glr_distill_args* a, void* stream) {
    const char* who = "glr_distill_loss";
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_logits(who, a->rows, a->vocab, a->logits, a->ld_logits, a->dlogits, a->ld_dlogits, a->weight, a->loss, a->dtype))
        return rc;
    if (a->topk < 0 || a->topk > GLR_MAX_TOPK) return refuse("%s: need 0 <= topk <= %d", who, GLR_MAX_TOPK);
    if (!dtype_ok(a->teacher_dtype)) return refuse("%s: unknown teacher_dtype %d", who, a->teacher_dtype);
    if (!flag(a->ids_index64) || !flag(a->labels_index64)) return refuse("%s: index64 must be 0 or 1", who);
    if (!matrix_ok(a->teacher, a->ld_teacher, a->rows, a->topk, a->teacher_dtype))
        return refuse("%s: teacher null, misaligned or with ld < topk", who);
    if (a->rows && a->topk && (!a->ids || (a->rows > 1 && a->ld_ids < a->topk) || !optional_ok(a->ids, a->ids_index64 ? 8 : 4)))
        return refuse("%s: ids null, misaligned or with ld < topk", who);
    if (!optional_ok(a->labels, a->labels_index64 ? 8 : 4)) return refuse("%s: labels misaligned", who);
    if (!vector_ok(a->row_loss, a->rows, 4)) return refuse("%s: row_loss is null or misaligned", who);
    if (!positive(a->temperature)) return refuse("%s: need a finite temperature > 0", who);
    if (!finite(a->soft) || !finite(a->hard)) return refuse("%s: soft and hard must be finite", who);
    loss::RowArgs r{};
    r.rows = a->rows; r.vocab = a->vocab; r.z = a->logits; r.ldz = a->ld_logits; r.dz = a->dlogits; r.lddz = a->ld_dlogits;
    r.weight = a->weight; r.share = a->rows ? static_cast<float>(1.0 / static_cast<double>(a->rows)) : 0.f;
    r.inv_tau = static_cast<float>(1.0 / static_cast<double>(a->temperature));
    r.row_loss = a->row_loss;
    r.teacher = a->teacher; r.ldt = a->ld_teacher; r.teacher_bf16 = a->teacher_dtype == GLR_BF16;
    r.ids = {a->ids, a->ids_index64}; r.ldi = a->ld_ids; r.topk = static_cast<int>(a->topk);
    r.labels = {a->labels, a->labels_index64};
    r.soft = a->soft; r.hard = a->hard;
    if (!(r.err = gave_up_counter())) return launched(who, cudaErrorNoDevice);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = loss::distill(r, a->dtype, st);
    if (e == cudaSuccess) e = loss::total(r.row_loss, r.weight, r.share, r.rows, a->loss, st);
    return launched(who, e);
}

extern "C" int glr_policy_loss(const glr_policy_args* a, void* stream) {
    const char* who = "glr_policy_loss";
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_logits(who, a->rows, a->vocab, a->logits, a->ld_logits, a->dlogits, a->ld_dlogits, a->weight, a->loss, a->dtype))
        return rc;
    if (!flag(a->index64)) return refuse("%s: index64 must be 0 or 1", who);
    if (!vector_ok(a->tokens, a->rows, a->index64 ? 8 : 4)) return refuse("%s: tokens is null or misaligned", who);
    if (!vector_ok(a->old_logp, a->rows, 4) || !vector_ok(a->advantage, a->rows, 4))
        return refuse("%s: old_logp or advantage is null or misaligned", who);
    if (!optional_ok(a->ref_logp, 4)) return refuse("%s: ref_logp misaligned", who);
    if (!vector_ok(a->row_loss, a->rows, 4) || !vector_ok(a->logp, a->rows, 4))
        return refuse("%s: row_loss or logp is null or misaligned", who);
    if (!positive(a->temperature)) return refuse("%s: need a finite temperature > 0", who);
    if (!finite(a->kl) || !(a->clip_low >= 0.f) || !finite(a->clip_low) || !(a->clip_high >= 0.f) || !finite(a->clip_high))
        return refuse("%s: need finite clip_low, clip_high >= 0 and a finite kl", who);
    loss::RowArgs r{};
    r.rows = a->rows; r.vocab = a->vocab; r.z = a->logits; r.ldz = a->ld_logits; r.dz = a->dlogits; r.lddz = a->ld_dlogits;
    r.weight = a->weight; r.share = a->rows ? static_cast<float>(1.0 / static_cast<double>(a->rows)) : 0.f;
    r.inv_tau = static_cast<float>(1.0 / static_cast<double>(a->temperature));
    r.row_loss = a->row_loss; r.logp = a->logp;
    r.tokens = {a->tokens, a->index64};
    r.old_logp = a->old_logp; r.advantage = a->advantage; r.ref_logp = a->ref_logp;
    r.clip_lo = static_cast<float>(1.0 - static_cast<double>(a->clip_low));
    r.clip_hi = static_cast<float>(1.0 + static_cast<double>(a->clip_high));
    r.kl = a->kl;
    if (!(r.err = gave_up_counter())) return launched(who, cudaErrorNoDevice);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = loss::policy(r, a->dtype, st);
    if (e == cudaSuccess) e = loss::total(r.row_loss, r.weight, r.share, r.rows, a->loss, st);
    return launched(who, e);
}

extern "C" int glr_preference_loss(const glr_preference_args* a, void* stream) {
    const char* who = "glr_preference_loss";
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_logits(who, a->rows, a->vocab, a->logits, a->ld_logits, a->dlogits, a->ld_dlogits, a->weight, a->loss, a->dtype))
        return rc;
    if (a->pairs < 0 || a->pairs > (int64_t(1) << 24)) return refuse("%s: need 0 <= pairs <= 2^24", who);
    if (!flag(a->tokens_index64) || !flag(a->offsets_index64) || !flag(a->average))
        return refuse("%s: index64 and average must be 0 or 1", who);
    if (a->kind != GLR_PREF_SIGMOID && a->kind != GLR_PREF_IPO) return refuse("%s: unknown kind %d", who, a->kind);
    if (!vector_ok(a->tokens, a->rows, a->tokens_index64 ? 8 : 4)) return refuse("%s: tokens is null or misaligned", who);
    if (!vector_ok(a->offsets, a->pairs, a->offsets_index64 ? 8 : 4)) return refuse("%s: offsets is null or misaligned", who);
    if (!optional_ok(a->ref_logp, 4)) return refuse("%s: ref_logp misaligned", who);
    if (!vector_ok(a->pair_loss, a->pairs, 4) || !vector_ok(a->seq_logp, a->pairs, 4) || !vector_ok(a->row_logp, a->rows, 4))
        return refuse("%s: pair_loss, seq_logp or row_logp is null or misaligned", who);
    if (!positive(a->beta)) return refuse("%s: need a finite beta > 0", who);
    if (!(a->smoothing >= 0.f && a->smoothing <= 1.f)) return refuse("%s: need 0 <= smoothing <= 1", who);
    if (!a->workspace || reinterpret_cast<uintptr_t>(a->workspace) % 16 ||
        a->workspace_bytes < GLR_PREFERENCE_WORKSPACE(a->rows, a->pairs))
        return refuse("%s: workspace is null, not 16-byte aligned or smaller than %lld bytes", who,
                      static_cast<long long>(GLR_PREFERENCE_WORKSPACE(a->rows, a->pairs)));
    loss::RowArgs r{};
    r.rows = a->rows; r.vocab = a->vocab; r.z = a->logits; r.ldz = a->ld_logits; r.dz = a->dlogits; r.lddz = a->ld_dlogits;
    r.inv_tau = 1.f;
    r.tokens = {a->tokens, a->tokens_index64};
    r.logp = a->row_logp;
    r.sums = static_cast<loss::RowSum*>(a->workspace);
    if (!(r.err = gave_up_counter())) return launched(who, cudaErrorNoDevice);
    loss::PairArgs p{};
    p.rows = a->rows; p.pairs = a->pairs; p.offsets = {a->offsets, a->offsets_index64};
    p.row_logp = r.logp; p.sums = r.sums; p.ref_logp = a->ref_logp; p.weight = a->weight;
    p.share = a->pairs ? static_cast<float>(1.0 / static_cast<double>(a->pairs)) : 0.f;
    p.beta = a->beta; p.smoothing = a->smoothing; p.kind = a->kind; p.average = a->average;
    p.pair_loss = a->pair_loss; p.seq_logp = a->seq_logp;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = loss::log_prob(r, a->dtype, st);
    if (e == cudaSuccess) e = loss::pairs(p, st);
    if (e == cudaSuccess && r.dz) e = loss::log_prob_grad(r, a->dtype, st);
    if (e == cudaSuccess) e = loss::total(p.pair_loss, p.weight, p.share, p.pairs, a->loss, st);
    return launched(who, e);
}

extern "C" int glr_operator_status(int32_t* gave_up) {
    if (gave_up) *gave_up = 0;
    int* p = gave_up_counter();
    int v = 0;
    if (!p) return launched("glr_operator_status", cudaErrorNoDevice);
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&v, p, sizeof(v), cudaMemcpyDeviceToHost);
    if (e != cudaSuccess) return launched("glr_operator_status", e);
    if (gave_up) *gave_up = v;
    if (v) {
        if ((e = cudaMemset(p, 0, sizeof(v))) != cudaSuccess) return launched("glr_operator_status", e);      // reported now
        set_global_error("a bounded wait in an operator's kernel gave up");
        return GLR_ETIMEOUT;
    }
    return GLR_OK;
}
