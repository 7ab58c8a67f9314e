// Entry points of the row operators around the step: embeddings, norms, 8-bit checkpoints of activations and token
// log-probabilities.  They check their arguments, fill the kernels' arguments and launch; nothing is kept between calls and
// nothing is allocated.
#include <algorithm>

#include "glr_checks.cuh"
#include "glr_linear.cuh"
#include "glr_rows.cuh"

using namespace glr;

namespace {

constexpr int64_t kMost = int64_t(1) << 30;

int check_nodes(const char* who, int64_t nodes, int64_t rows) {
    if (nodes < 1 || nodes > GLR_MAX_NODES) return refuse("%s: need 1 <= nodes <= %d", who, GLR_MAX_NODES);
    if (rows < 0 || rows > kMost / nodes) return refuse("%s: need 0 <= nodes * rows <= 2^30", who);
    return GLR_OK;
}
int check_workspace(const char* who, const void* p, int64_t bytes, int64_t need) {
    if (need > 0 && (!p || reinterpret_cast<uintptr_t>(p) % 16 || bytes < need))
        return refuse("%s: workspace is null, not 16-byte aligned or smaller than %lld bytes", who, static_cast<long long>(need));
    return GLR_OK;
}
bool codes_ok(const void* codes, int64_t ldc, const void* scales, int64_t lds, int64_t rows, int64_t cols) {
    if (rows == 0 || cols == 0) return true;
    return codes && scales && (rows == 1 || (ldc >= cols && lds >= (cols + 31) / 32));
}
// Two nodes' gradients in one place would be written by both at once.
bool apart(void* const* p, int64_t n) {
    for (int64_t i = 1; i < n; ++i)
        for (int64_t j = 0; j < i; ++j)
            if (p[i] == p[j] && p[i]) return false;
    return true;
}
// An output in the place of an input: the same rows, or none of them.
bool in_place_ok(const void* out, int64_t ldo, const void* in, int64_t ldi, int64_t rows) { return !out || out != in || rows <= 1 || ldo == ldi; }

int check_pack(const char* who, int64_t rows, int64_t cols, int dtype) {
    if (!dtype_ok(dtype)) return refuse("%s: unknown dtype %d", who, dtype);
    if (rows < 0 || rows > kMost || cols < 0 || cols > (int64_t(1) << 24)) return refuse("%s: need 0 <= rows <= 2^30 and 0 <= cols <= 2^24", who);
    return GLR_OK;
}

int check_embedding_grad(const char* who, const glr_embedding_grad_args* a) {
    if (!a) return refuse("%s: null arguments", who);
    if (!dtype_ok(a->dtype)) return refuse("%s: unknown dtype %d", who, a->dtype);
    if (!dtype_ok(a->grad_dtype)) return refuse("%s: unknown grad_dtype %d", who, a->grad_dtype);
    if (!flag(a->index64) || !flag(a->accumulate)) return refuse("%s: index64 and accumulate must be 0 or 1", who);
    if (int rc = check_nodes(who, a->nodes, a->rows)) return rc;
    if (a->vocab < 0 || a->vocab >= (int64_t(1) << 24) || a->d < 0 || a->d > (int64_t(1) << 20))
        return refuse("%s: need 0 <= vocab < 2^24 and 0 <= d <= 2^20", who);
    if (!finite(a->scale)) return refuse("%s: scale must be finite", who);
    const int64_t all = a->nodes * a->rows;
    if (!matrix_ok(a->dY, a->lddy, all, a->d, a->dtype)) return refuse("%s: dY null, misaligned or with ld < d", who);
    if (!vector_ok(a->tokens, all, a->index64 ? 8 : 4)) return refuse("%s: tokens is null or misaligned", who);
    if (!a->dE) return refuse("%s: dE is null", who);
    for (int64_t i = 0; i < a->nodes; ++i)
        if (!vector_ok(a->dE[i], a->vocab * a->d, bytes_of(a->grad_dtype))) return refuse("%s: dE[%d] is null or misaligned", who, (int)i);
    if (!apart(a->dE, a->nodes)) return refuse("%s: the same dE twice", who);
    return GLR_OK;
}
int64_t embedding_grad_need(const glr_embedding_grad_args* a) {
    return a->vocab && a->d ? rows::embedding_grad_bytes(a->nodes, a->rows, a->vocab, a->d) : 0;
}

int check_norm_grad(const char* who, const glr_norm_grad_args* a) {
    if (!a) return refuse("%s: null arguments", who);
    if (!dtype_ok(a->dtype)) return refuse("%s: unknown dtype %d", who, a->dtype);
    if (!dtype_ok(a->grad_dtype)) return refuse("%s: unknown grad_dtype %d", who, a->grad_dtype);
    if (int rc = check_nodes(who, a->nodes, a->rows)) return rc;
    if (a->n < 1 || a->n > GLR_MAX_NORM) return refuse("%s: need 1 <= n <= %d", who, GLR_MAX_NORM);
    const int64_t all = a->nodes * a->rows;
    if (!matrix_ok(a->dY, a->lddy, all, a->n, a->dtype)) return refuse("%s: dY null, misaligned or with ld < n", who);
    if (!matrix_ok(a->H, a->ldh, all, a->n, a->dtype)) return refuse("%s: H null, misaligned or with ld < n", who);
    if (!vector_ok(a->rstd, all, 4)) return refuse("%s: rstd is null or misaligned", who);
    if (!optional_ok(a->weight, bytes_of(a->dtype))) return refuse("%s: weight misaligned", who);
    if (a->residual && !matrix_ok(a->residual, a->ldr, all, a->n, a->dtype)) return refuse("%s: residual misaligned or with ld < n", who);
    if (a->dX && !matrix_ok(a->dX, a->lddx, all, a->n, a->dtype)) return refuse("%s: dX misaligned or with ld < n", who);
    if (!in_place_ok(a->dX, a->lddx, a->residual, a->ldr, all) || !in_place_ok(a->dX, a->lddx, a->dY, a->lddy, all))
        return refuse("%s: dX in place of dY or residual needs the same ld", who);
    if (a->dX && a->dX == a->H && all) return refuse("%s: dX must not be H", who);
    for (int64_t i = 0; a->dweight && i < a->nodes; ++i)
        if (!vector_ok(a->dweight[i], a->n, bytes_of(a->grad_dtype))) return refuse("%s: dweight[%d] is null or misaligned", who, (int)i);
    if (a->dweight && !apart(a->dweight, a->nodes)) return refuse("%s: the same dweight twice", who);
    return GLR_OK;
}
int64_t norm_grad_need(const glr_norm_grad_args* a) {
    return a->dweight ? rows::norm_grad_bytes(a->nodes, a->rows, static_cast<int>(a->n)) : 0;
}

// The checkpoint's gradient in its workspace: the layer's input, and what the products ask for.
struct CheckpointPlan {
    int64_t ld, plane, inner;
    int64_t bytes() const { return plane + inner; }
};
glr_linear_grad_input_args input_args(const glr_linear_grad_checkpoint_args* a) {
    glr_linear_grad_input_args g{};
    g.rows = a->nodes * a->rows; g.n = a->n; g.k = a->k;
    g.dZ = a->dZ; g.lddz = a->lddz; g.W = a->W; g.ldw = a->ldw;
    g.dX = a->dX; g.lddx = a->lddx; g.residual = a->residual; g.ldr = a->ldr;
    g.dtype = a->dtype;
    return g;
}
glr_linear_grad_weight_args weight_args(const glr_linear_grad_checkpoint_args* a, const void* x, int64_t ldx) {
    glr_linear_grad_weight_args g{};
    g.nodes = a->nodes; g.rows = a->rows; g.n = a->n; g.k = a->k;
    g.dZ = a->dZ; g.lddz = a->lddz; g.X = x; g.ldx = ldx;
    g.dW = a->dW; g.db = a->db;
    g.dtype = a->dtype; g.grad_dtype = a->grad_dtype;
    return g;
}
int plan_checkpoint(const char* who, const glr_linear_grad_checkpoint_args* a, CheckpointPlan& p) {
    if (!a) return refuse("%s: null arguments", who);
    if (!dtype_ok(a->dtype)) return refuse("%s: unknown dtype %d", who, a->dtype);
    if (!dtype_ok(a->grad_dtype)) return refuse("%s: unknown grad_dtype %d", who, a->grad_dtype);
    if (a->act < GLR_ACT_NONE || a->act > GLR_ACT_SILU) return refuse("%s: unknown activation %d", who, a->act);
    if (int rc = check_nodes(who, a->nodes, a->rows)) return rc;
    if (a->n < 0 || a->n > (int64_t(1) << 24) || a->k < 0 || a->k > (int64_t(1) << 24)) return refuse("%s: need 0 <= n, k <= 2^24", who);
    if (!a->dW && !a->dX) return refuse("%s: neither dW nor dX is wanted", who);
    if (a->db && !a->dW) return refuse("%s: db needs dW", who);
    const int64_t all = a->nodes * a->rows, es = bytes_of(a->dtype), gs = bytes_of(a->grad_dtype);
    if (!matrix_ok(a->dZ, a->lddz, all, a->n, a->dtype)) return refuse("%s: dZ null, misaligned or with ld < n", who);
    if ((a->dW || a->act != GLR_ACT_NONE) && !codes_ok(a->codes, a->ld_codes, a->scales, a->ld_scales, all, a->k))
        return refuse("%s: codes or scales null or with ld < their columns", who);
    if (a->dX) {
        if (!matrix_ok(a->W, a->ldw, a->n, a->k, a->dtype)) return refuse("%s: W null, misaligned or with ld < k", who);
        if (!matrix_ok(a->dX, a->lddx, all, a->k, a->dtype)) return refuse("%s: dX misaligned or with ld < k", who);
        if (a->residual && !matrix_ok(a->residual, a->ldr, all, a->k, a->dtype)) return refuse("%s: residual misaligned or with ld < k", who);
        if (!in_place_ok(a->dX, a->lddx, a->residual, a->ldr, all)) return refuse("%s: residual in place of dX needs the same ld", who);
    }
    for (int64_t i = 0; a->dW && i < a->nodes; ++i) {
        if (!vector_ok(a->dW[i], a->n * a->k, gs)) return refuse("%s: dW[%d] is null or misaligned", who, (int)i);
        if (a->db && !vector_ok(a->db[i], a->n, gs)) return refuse("%s: db[%d] is null or misaligned", who, (int)i);
    }
    if ((a->dW && !apart(a->dW, a->nodes)) || (a->db && !apart(a->db, a->nodes))) return refuse("%s: the same dW or db twice", who);
    // rows on 16 bytes, as the products want them; the query's pointer only tells it so
    p.ld = (a->k + 7) / 8 * 8;
    p.plane = a->dW ? (all * p.ld * es + 255) / 256 * 256 : 0;
    p.inner = 0;
    int64_t need = 0;
    if (a->dX) {
        const glr_linear_grad_input_args g = input_args(a);
        if (int rc = glr_linear_grad_input_workspace(&g, &need)) return rc;
        p.inner = std::max(p.inner, need);
    }
    if (a->dW) {
        const glr_linear_grad_weight_args g = weight_args(a, reinterpret_cast<const void*>(uintptr_t(256)), p.ld);
        if (int rc = glr_linear_grad_weight_workspace(&g, &need)) return rc;
        p.inner = std::max(p.inner, need);
    }
    return GLR_OK;
}

}  // namespace

extern "C" int glr_embedding(const glr_embedding_args* a, void* stream) {
    const char* who = "glr_embedding";
    if (!a) return refuse("%s: null arguments", who);
    if (!dtype_ok(a->dtype)) return refuse("%s: unknown dtype %d", who, a->dtype);
    if (!flag(a->index64)) return refuse("%s: index64 must be 0 or 1", who);
    if (a->rows < 0 || a->rows > kMost || a->vocab < 0 || a->vocab >= (int64_t(1) << 24) || a->d < 0 || a->d > (int64_t(1) << 20))
        return refuse("%s: need 0 <= rows <= 2^30, 0 <= vocab < 2^24 and 0 <= d <= 2^20", who);
    if (!finite(a->scale)) return refuse("%s: scale must be finite", who);
    if (!matrix_ok(a->E, a->lde, a->vocab, a->d, a->dtype)) return refuse("%s: E null, misaligned or with ld < d", who);
    if (!matrix_ok(a->Y, a->ldy, a->rows, a->d, a->dtype)) return refuse("%s: Y null, misaligned or with ld < d", who);
    if (!vector_ok(a->tokens, a->rows, a->index64 ? 8 : 4)) return refuse("%s: tokens is null or misaligned", who);
    rows::Lookup l{};
    l.rows = a->rows; l.vocab = a->vocab; l.d = a->d; l.E = a->E; l.lde = a->lde; l.tokens = {a->tokens, a->index64};
    l.Y = a->Y; l.ldy = a->ldy; l.scale = a->scale;
    return launched(who, rows::lookup(l, a->dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_embedding_grad_workspace(const glr_embedding_grad_args* a, int64_t* bytes) {
    const char* who = "glr_embedding_grad_workspace";
    if (!bytes) return refuse("%s: bytes is null", who);
    if (int rc = check_embedding_grad(who, a)) return rc;
    *bytes = embedding_grad_need(a);
    return GLR_OK;
}
extern "C" int glr_embedding_grad(const glr_embedding_grad_args* a, void* stream) {
    const char* who = "glr_embedding_grad";
    if (int rc = check_embedding_grad(who, a)) return rc;
    if (int rc = check_workspace(who, a->workspace, a->workspace_bytes, embedding_grad_need(a))) return rc;
    rows::EmbeddingGrad g{};
    g.nodes = a->nodes; g.rows = a->rows; g.vocab = a->vocab; g.d = a->d; g.dY = a->dY; g.lddy = a->lddy;
    g.tokens = {a->tokens, a->index64}; g.scale = a->scale; g.accumulate = a->accumulate; g.workspace = a->workspace;
    for (int64_t i = 0; i < a->nodes; ++i) g.dE[i] = a->dE[i];
    return launched(who, rows::embedding_grad(g, a->dtype, a->grad_dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_norm(const glr_norm_args* a, void* stream) {
    const char* who = "glr_norm";
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_pack(who, a->rows, 1, a->dtype)) return rc;
    if (a->n < 1 || a->n > GLR_MAX_NORM) return refuse("%s: need 1 <= n <= %d", who, GLR_MAX_NORM);
    if (!positive(a->eps)) return refuse("%s: need a finite eps >= 1.2e-38", who);
    if (!matrix_ok(a->X, a->ldx, a->rows, a->n, a->dtype)) return refuse("%s: X null, misaligned or with ld < n", who);
    if ((a->residual && !matrix_ok(a->residual, a->ldr, a->rows, a->n, a->dtype)) || (a->H && !matrix_ok(a->H, a->ldh, a->rows, a->n, a->dtype)) ||
        (a->Y && !matrix_ok(a->Y, a->ldy, a->rows, a->n, a->dtype)))
        return refuse("%s: residual, H or Y misaligned or with ld < n", who);
    if (!optional_ok(a->weight, bytes_of(a->dtype)) || !optional_ok(a->rstd, 4)) return refuse("%s: weight or rstd misaligned", who);
    if (!a->codes != !a->scales) return refuse("%s: codes and scales go together", who);
    if (a->codes && !codes_ok(a->codes, a->ld_codes, a->scales, a->ld_scales, a->rows, a->n))
        return refuse("%s: codes or scales with ld < their columns", who);
    if (a->H && a->H == a->Y && a->rows) return refuse("%s: H and Y must not be one matrix", who);
    if (!in_place_ok(a->H, a->ldh, a->X, a->ldx, a->rows) || !in_place_ok(a->H, a->ldh, a->residual, a->ldr, a->rows) ||
        !in_place_ok(a->Y, a->ldy, a->X, a->ldx, a->rows) || !in_place_ok(a->Y, a->ldy, a->residual, a->ldr, a->rows))
        return refuse("%s: H or Y in place of X or residual needs the same ld", who);
    rows::Norm m{};
    m.rows = a->rows; m.n = static_cast<int>(a->n); m.X = a->X; m.ldx = a->ldx; m.residual = a->residual; m.ldr = a->ldr;
    m.weight = a->weight; m.H = a->H; m.ldh = a->ldh; m.Y = a->Y; m.ldy = a->ldy; m.rstd = a->rstd;
    m.codes = static_cast<int8_t*>(a->codes); m.ld_codes = a->ld_codes;
    m.scales = static_cast<uint8_t*>(a->scales); m.ld_scales = a->ld_scales; m.eps = a->eps;
    return launched(who, rows::norm(m, a->dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_norm_grad_workspace(const glr_norm_grad_args* a, int64_t* bytes) {
    const char* who = "glr_norm_grad_workspace";
    if (!bytes) return refuse("%s: bytes is null", who);
    if (int rc = check_norm_grad(who, a)) return rc;
    *bytes = norm_grad_need(a);
    return GLR_OK;
}
extern "C" int glr_norm_grad(const glr_norm_grad_args* a, void* stream) {
    const char* who = "glr_norm_grad";
    if (int rc = check_norm_grad(who, a)) return rc;
    if (!a->dX && !a->dweight) return GLR_OK;
    if (int rc = check_workspace(who, a->workspace, a->workspace_bytes, norm_grad_need(a))) return rc;
    rows::NormGrad g{};
    g.nodes = a->nodes; g.rows = a->rows; g.n = static_cast<int>(a->n); g.dY = a->dY; g.lddy = a->lddy; g.H = a->H; g.ldh = a->ldh;
    g.rstd = a->rstd; g.weight = a->weight; g.residual = a->residual; g.ldr = a->ldr; g.dX = a->dX; g.lddx = a->lddx;
    g.want_dweight = a->dweight != nullptr; g.partial = static_cast<float*>(a->workspace);
    for (int64_t i = 0; a->dweight && i < a->nodes; ++i) g.dweight[i] = a->dweight[i];
    return launched(who, rows::norm_grad(g, a->dtype, a->grad_dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_checkpoint_pack(const glr_checkpoint_pack_args* a, void* stream) {
    const char* who = "glr_checkpoint_pack";
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_pack(who, a->rows, a->cols, a->dtype)) return rc;
    if (!matrix_ok(a->X, a->ldx, a->rows, a->cols, a->dtype)) return refuse("%s: X null, misaligned or with ld < cols", who);
    if (!codes_ok(a->codes, a->ld_codes, a->scales, a->ld_scales, a->rows, a->cols))
        return refuse("%s: codes or scales null or with ld < their columns", who);
    rows::Pack p{};
    p.rows = a->rows; p.cols = a->cols; p.X = a->X; p.ldx = a->ldx;
    p.codes = static_cast<int8_t*>(a->codes); p.ld_codes = a->ld_codes;
    p.scales = static_cast<uint8_t*>(a->scales); p.ld_scales = a->ld_scales;
    return launched(who, rows::pack(p, a->dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_checkpoint_unpack(const glr_checkpoint_unpack_args* a, void* stream) {
    const char* who = "glr_checkpoint_unpack";
    if (!a) return refuse("%s: null arguments", who);
    if (int rc = check_pack(who, a->rows, a->cols, a->dtype)) return rc;
    if (a->act < GLR_ACT_NONE || a->act > GLR_ACT_SILU) return refuse("%s: unknown activation %d", who, a->act);
    if (!codes_ok(a->codes, a->ld_codes, a->scales, a->ld_scales, a->rows, a->cols))
        return refuse("%s: codes or scales null or with ld < their columns", who);
    if (!matrix_ok(a->Y, a->ldy, a->rows, a->cols, a->dtype)) return refuse("%s: Y null, misaligned or with ld < cols", who);
    rows::Unpack u{};
    u.rows = a->rows; u.cols = a->cols;
    u.codes = static_cast<const int8_t*>(a->codes); u.ld_codes = a->ld_codes;
    u.scales = static_cast<const uint8_t*>(a->scales); u.ld_scales = a->ld_scales;
    u.Y = a->Y; u.ldy = a->ldy; u.act = a->act;
    return launched(who, rows::unpack(u, a->dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_linear_grad_checkpoint_workspace(const glr_linear_grad_checkpoint_args* a, int64_t* bytes) {
    const char* who = "glr_linear_grad_checkpoint_workspace";
    CheckpointPlan p{};
    if (!bytes) return refuse("%s: bytes is null", who);
    if (int rc = plan_checkpoint(who, a, p)) return rc;
    *bytes = p.bytes();
    return GLR_OK;
}
extern "C" int glr_linear_grad_checkpoint(const glr_linear_grad_checkpoint_args* a, void* stream) {
    const char* who = "glr_linear_grad_checkpoint";
    CheckpointPlan p{};
    if (int rc = plan_checkpoint(who, a, p)) return rc;
    if (int rc = check_workspace(who, a->workspace, a->workspace_bytes, p.bytes())) return rc;
    const int8_t* codes = static_cast<const int8_t*>(a->codes);
    const uint8_t* scales = static_cast<const uint8_t*>(a->scales);
    uint8_t* space = static_cast<uint8_t*>(a->workspace);
    void* inner = p.inner ? space + p.plane : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dX) {
        glr_linear_grad_input_args g = input_args(a);
        g.workspace = inner; g.workspace_bytes = p.inner;
        if (int rc = linear::grad_input_packed(who, g, codes, a->ld_codes, scales, a->ld_scales, a->act, st)) return rc;
    }
    if (a->dW) {
        // (The epilogue of dX, which has the pre-activation in hand, could write it too: 8192 x 5632 to 2048 bf16 with SiLU, 318 us, took
        // 7 us more so, and other input gradients 8.)
        rows::Unpack u{};
        u.rows = a->nodes * a->rows; u.cols = a->k;
        u.codes = codes; u.ld_codes = a->ld_codes; u.scales = scales; u.ld_scales = a->ld_scales;
        u.Y = space; u.ldy = p.ld; u.act = a->act;
        if (int rc = launched(who, rows::unpack(u, a->dtype, st))) return rc;
        glr_linear_grad_weight_args g = weight_args(a, space, p.ld);
        g.workspace = inner; g.workspace_bytes = p.inner;
        if (int rc = glr_linear_grad_weight(&g, stream)) return rc;
    }
    return GLR_OK;
}

extern "C" int glr_token_logp(const glr_token_logp_args* a, void* stream) {
    const char* who = "glr_token_logp";
    if (!a) return refuse("%s: null arguments", who);
    if (!dtype_ok(a->dtype)) return refuse("%s: unknown dtype %d", who, a->dtype);
    if (a->rows < 0 || a->rows > kMaxRows) return refuse("%s: need 0 <= rows <= 2^24", who);
    if (a->vocab < 1 || a->vocab > GLR_MAX_LOGIT_BYTES || a->vocab * bytes_of(a->dtype) > GLR_MAX_LOGIT_BYTES)
        return refuse("%s: need vocab >= 1 and rows of logits of at most %d bytes", who, GLR_MAX_LOGIT_BYTES);
    if (a->topk < 0 || a->topk > GLR_MAX_TOPK) return refuse("%s: need 0 <= topk <= %d", who, GLR_MAX_TOPK);
    if (!flag(a->tokens_index64) || !flag(a->ids_index64)) return refuse("%s: index64 must be 0 or 1", who);
    if (!matrix_ok(a->logits, a->ld_logits, a->rows, a->vocab, a->dtype)) return refuse("%s: logits null, misaligned or with ld < vocab", who);
    if (!optional_ok(a->tokens, a->tokens_index64 ? 8 : 4) || (a->logp && !a->tokens && a->rows)) return refuse("%s: tokens misaligned, or null with logp", who);
    if (!optional_ok(a->logp, 4) || !optional_ok(a->lse, 4) || !optional_ok(a->entropy, 4)) return refuse("%s: logp, lse or entropy misaligned", who);
    if (!optional_ok(a->top_logp, 4) || (a->top_logp && a->rows > 1 && a->ld_top_logp < a->topk))
        return refuse("%s: top_logp misaligned or with ld < topk", who);
    if (!optional_ok(a->top_ids, a->ids_index64 ? 8 : 4) || (a->top_ids && a->rows > 1 && a->ld_top_ids < a->topk))
        return refuse("%s: top_ids misaligned or with ld < topk", who);
    if (!positive(a->temperature)) return refuse("%s: need a finite temperature > 0", who);
    rows::TokenLogp t{};
    t.rows = a->rows; t.vocab = a->vocab; t.topk = a->top_logp || a->top_ids ? static_cast<int>(a->topk) : 0;
    t.z = a->logits; t.ldz = a->ld_logits; t.tokens = {a->tokens, a->tokens_index64};
    t.logp = a->logp; t.lse = a->lse; t.entropy = a->entropy;
    t.top_logp = a->top_logp; t.ld_top_logp = a->ld_top_logp; t.top_ids = a->top_ids; t.ld_top_ids = a->ld_top_ids; t.ids_wide = a->ids_index64;
    t.inv_tau = static_cast<float>(1.0 / static_cast<double>(a->temperature));
    return launched(who, rows::token_logp(t, a->dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" int glr_token_logp_grad(const glr_token_logp_grad_args* a, void* stream) {
    const char* who = "glr_token_logp_grad";
    if (!a) return refuse("%s: null arguments", who);
    if (!dtype_ok(a->dtype)) return refuse("%s: unknown dtype %d", who, a->dtype);
    if (a->rows < 0 || a->rows > kMaxRows) return refuse("%s: need 0 <= rows <= 2^24", who);
    if (a->vocab < 1 || a->vocab > GLR_MAX_LOGIT_BYTES || a->vocab * bytes_of(a->dtype) > GLR_MAX_LOGIT_BYTES)
        return refuse("%s: need vocab >= 1 and rows of logits of at most %d bytes", who, GLR_MAX_LOGIT_BYTES);
    if (!flag(a->index64)) return refuse("%s: index64 must be 0 or 1", who);
    if (!matrix_ok(a->logits, a->ld_logits, a->rows, a->vocab, a->dtype)) return refuse("%s: logits null, misaligned or with ld < vocab", who);
    if (!matrix_ok(a->dlogits, a->ld_dlogits, a->rows, a->vocab, a->dtype)) return refuse("%s: dlogits null, misaligned or with ld < vocab", who);
    if (!in_place_ok(a->dlogits, a->ld_dlogits, a->logits, a->ld_logits, a->rows)) return refuse("%s: dlogits in place of logits needs the same ld", who);
    if (!vector_ok(a->lse, a->rows, 4)) return refuse("%s: lse is null or misaligned", who);
    if (!optional_ok(a->dlogp, 4) || !optional_ok(a->tokens, a->index64 ? 8 : 4) || (a->dlogp && !a->tokens && a->rows))
        return refuse("%s: dlogp or tokens misaligned, or dlogp without tokens", who);
    if (!optional_ok(a->dentropy, 4) || !optional_ok(a->entropy, 4) || (a->dentropy && !a->entropy && a->rows))
        return refuse("%s: dentropy or entropy misaligned, or dentropy without entropy", who);
    if (!positive(a->temperature)) return refuse("%s: need a finite temperature > 0", who);
    rows::TokenLogpGrad g{};
    g.rows = a->rows; g.vocab = a->vocab; g.z = a->logits; g.ldz = a->ld_logits; g.tokens = {a->tokens, a->index64};
    g.lse = a->lse; g.entropy = a->entropy; g.dlogp = a->dlogp; g.dentropy = a->dentropy; g.dz = a->dlogits; g.lddz = a->ld_dlogits;
    g.inv_tau = static_cast<float>(1.0 / static_cast<double>(a->temperature));
    return launched(who, rows::token_logp_grad(g, a->dtype, static_cast<cudaStream_t>(stream)));
}
