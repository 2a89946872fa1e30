// extern "C" boundary: argument checks, then dispatch to the kernel launchers.  See include/onecomp.h.
#include "common.hpp"
#include "attention.hpp"
#include "block.hpp"
#include <cmath>
#include <initializer_list>
#include <dlfcn.h>
#include <cstdlib>

using namespace onecomp;

namespace {
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Named host ranges around the entry points for a profiler's marker trace (rocprofv3 --marker-trace), off unless the
// environment holds ONECOMP_ROCTX=1 when the first entry point is called: then the ROCTx library is looked up at run
// time (the library does not link against it) and every call pushes a range with its own name.  The launches are
// asynchronous, so a range covers the argument checks and the enqueueing, not the kernels' run time.
struct Roctx {
    int (*push)(const char*) = nullptr;
    int (*pop)() = nullptr;
};
const Roctx& roctx() {
    static const Roctx r = [] {
        Roctx x;
        const char* e = std::getenv("ONECOMP_ROCTX");
        if (!e || e[0] != '1' || e[1] != 0) return x;
        for (const char* lib : {"librocprofiler-sdk-roctx.so.1", "librocprofiler-sdk-roctx.so", "libroctx64.so.4", "libroctx64.so"}) {
            void* h = dlopen(lib, RTLD_NOW | RTLD_LOCAL);
            if (!h) continue;
            x.push = reinterpret_cast<int (*)(const char*)>(dlsym(h, "roctxRangePushA"));
            x.pop = reinterpret_cast<int (*)()>(dlsym(h, "roctxRangePop"));
            if (x.push && x.pop) return x;
            x = Roctx();
        }
        return x;
    }();
    return r;
}
struct ApiRange {
    const Roctx& r;
    explicit ApiRange(const char* name) : r(roctx()) { if (r.push) r.push(name); }
    ~ApiRange() { if (r.push) r.pop(); }
    ApiRange(const ApiRange&) = delete;
    ApiRange& operator=(const ApiRange&) = delete;
};

// ONECOMP_OK if a shape can be worked on; what its arrays hold is the kernels' business
onecomp_status check_attention(const onecomp_attention_shape* s) {
    if (!s) return ONECOMP_ERR_INVALID_ARG;
    if (s->dtype != ONECOMP_F32 && s->dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (s->n_heads <= 0 || s->n_kv_heads <= 0 || s->head_dim <= 0 || s->n_seqs < 0 || s->n_heads % s->n_kv_heads != 0)
        return ONECOMP_ERR_INVALID_ARG;
    if (s->head_dim > 128 || s->head_dim % (s->dtype == ONECOMP_BF16 ? 8 : 4) != 0 || s->n_heads > (1 << 16)) return ONECOMP_ERR_UNSUPPORTED;
    if (!(s->scale > 0.f) || !std::isfinite(s->scale)) return ONECOMP_ERR_INVALID_ARG;
    // scale log2(e) is a normal number, and so is a log-sum-exp over it, with which the gradients begin their scores
    if (s->scale < 0x1p-100f || s->scale > 0x1p100f) return ONECOMP_ERR_UNSUPPORTED;
    const int64_t most = (int64_t(1) << 31) - 4096;
    if (s->total_q < 0 || s->total_k < 0 || s->max_q < 0 || s->max_k < 0 || s->total_q > most || s->total_k > most || s->n_seqs > (1 << 24))
        return ONECOMP_ERR_INVALID_ARG;
    if (!s->cu_q || !s->cu_k) return ONECOMP_ERR_INVALID_ARG;
    return ONECOMP_OK;
}

bool check_heads(const onecomp_attention_shape* s, const onecomp_heads* h, int64_t rows) {
    if (!h) return false;
    if (rows == 0) return true;
    const int64_t esz = s->dtype == ONECOMP_BF16 ? 2 : 4;
    return h->data && aligned(h->data, 16) && h->token_stride >= s->head_dim && h->token_stride <= (1 << 22) && h->head_stride >= 0 &&
           h->head_stride <= (int64_t(1) << 40) && (h->token_stride * esz) % 16 == 0 && (h->head_stride * esz) % 16 == 0;
}

// whether two tensors begin at the same place; rows: 0 if either has none
bool same(const onecomp_heads* a, const onecomp_heads* b, int64_t rows) { return rows > 0 && a->data == b->data; }

onecomp_status check_norm(const onecomp_norm_shape* s) {
    if (!s) return ONECOMP_ERR_INVALID_ARG;
    if ((s->dtype != ONECOMP_F32 && s->dtype != ONECOMP_BF16) || (s->w_dtype != ONECOMP_F32 && s->w_dtype != ONECOMP_BF16)) return ONECOMP_ERR_UNSUPPORTED;
    if (s->kind != ONECOMP_NORM_RMS && s->kind != ONECOMP_NORM_LAYER) return ONECOMP_ERR_UNSUPPORTED;
    if (s->gate_kind != ONECOMP_GATE_NONE && s->gate_kind != ONECOMP_GATE_CHANNEL && s->gate_kind != ONECOMP_GATE_ROWS) return ONECOMP_ERR_UNSUPPORTED;
    if (s->rows < 0 || s->width <= 0 || s->rows > (int64_t(1) << 31) - 4096 || !(s->eps >= 0.f) || !std::isfinite(s->eps) || !std::isfinite(s->residual_scale))
        return ONECOMP_ERR_INVALID_ARG;
    if (s->width > 32768) return ONECOMP_ERR_UNSUPPORTED;
    return ONECOMP_OK;
}

// rows of the shape (NULL: fine, nothing is there)
bool check_rows(const onecomp_norm_shape* s, const onecomp_rows* r) {
    if (!r) return true;
    if (s->rows == 0) return true;
    return r->data && aligned(r->data, s->dtype == ONECOMP_BF16 ? 2 : 4) && r->row_stride >= s->width && r->row_stride <= (int64_t(1) << 31);
}
bool check_param(const onecomp_norm_shape* s, const void* p) { return aligned(p, s->w_dtype == ONECOMP_BF16 ? 2 : 4); }

// Results over inputs are written row by row as the rows are read: no other row may begin where the result's does.
bool apart_or_same(const onecomp_norm_shape* s, std::initializer_list<const onecomp_rows*> results, std::initializer_list<const onecomp_rows*> inputs) {
    if (s->rows == 0) return true;
    for (const onecomp_rows* r : results)
        for (const onecomp_rows* i : inputs)
            if (r && i && r->data == i->data && r->row_stride != i->row_stride && s->rows > 1) return false;
    for (const onecomp_rows* const* r = results.begin(); r != results.end(); ++r)
        for (const onecomp_rows* const* other = results.begin(); other != r; ++other)
            if (*r && *other && (*r)->data == (*other)->data) return false;
    return true;
}

block::Rows rows_of(const onecomp_rows* r) { return r ? block::Rows{r->data, r->row_stride} : block::Rows{nullptr, 0}; }

block::Params norm_params(const onecomp_norm_shape* s) {
    block::Params P{};
    P.rows = s->rows;
    P.width = int(s->width);
    P.layer = s->kind == ONECOMP_NORM_LAYER;
    P.post = s->post_norm != 0;
    P.gate_rows = s->gate_kind == ONECOMP_GATE_ROWS;
    P.w_bf16 = s->w_dtype == ONECOMP_BF16;
    P.scale = s->residual_scale;
    P.eps = s->eps;
    return P;
}

// what both directions have in common
onecomp_status norm_arguments(const onecomp_norm_shape* s, block::Params& P, const onecomp_rows* h, const onecomp_rows* y, const void* weight, const void* bias,
                              const void* post_weight, const void* post_bias, const onecomp_rows* gate) {
    if (!h || !check_rows(s, h) || !check_rows(s, y)) return ONECOMP_ERR_INVALID_ARG;
    if (!check_param(s, weight) || !check_param(s, bias) || !check_param(s, post_weight) || !check_param(s, post_bias)) return ONECOMP_ERR_INVALID_ARG;
    if ((!y && (s->post_norm || s->gate_kind != ONECOMP_GATE_NONE)) || (!s->post_norm && (post_weight || post_bias))) return ONECOMP_ERR_INVALID_ARG;
    if (s->kind == ONECOMP_NORM_RMS && (bias || post_bias)) return ONECOMP_ERR_INVALID_ARG;
    if ((s->gate_kind != ONECOMP_GATE_NONE) != (gate != nullptr)) return ONECOMP_ERR_INVALID_ARG;
    if (s->gate_kind == ONECOMP_GATE_ROWS && !check_rows(s, gate)) return ONECOMP_ERR_INVALID_ARG;
    if (s->gate_kind == ONECOMP_GATE_CHANNEL && (!gate->data || !check_param(s, gate->data))) return ONECOMP_ERR_INVALID_ARG;
    P = norm_params(s);
    P.h = rows_of(h);
    P.y = rows_of(y);
    P.gate = rows_of(gate);
    P.weight = weight;
    P.bias = bias;
    P.post_weight = post_weight;
    P.post_bias = post_bias;
    if (!y) P.scale = 1.f;                                        // h' is h
    return ONECOMP_OK;
}

attn::View view(const onecomp_heads* h) { return attn::View{h->data, h->token_stride, h->head_stride}; }

attn::Params attention_params(const onecomp_attention_shape* s) {
    attn::Params P{};
    P.cu_q = s->cu_q;
    P.cu_k = s->cu_k;
    P.len_k = s->len_k;
    P.total_q = s->total_q;
    P.total_k = s->total_k;
    P.n_seqs = s->n_seqs;
    P.heads = s->n_heads;
    P.kv_heads = s->n_kv_heads;
    P.group = s->n_heads / s->n_kv_heads;
    P.dim = s->head_dim;
    P.causal = s->causal != 0;
    P.scale = s->scale;
    P.c = s->scale * attn::LOG2E;
    // no sequence has more keys than all of them; more queries than there are still ask for the launch shape of so many
    P.max_q = s->max_q < (int64_t(1) << 31) ? s->max_q : int64_t(1) << 31;
    P.max_k = s->max_k < s->total_k ? s->max_k : s->total_k;
    return P;
}
}  // namespace

#define ONECOMP_API __attribute__((visibility("default")))
extern "C" {

ONECOMP_API size_t onecomp_accumulate_workspace_bytes(onecomp_dtype x_dtype, int64_t d_in) {
    if (x_dtype != ONECOMP_BF16 || d_in <= 0 || d_in % 16 != 0 || d_in > (1 << 20)) return 0;
    return gram_workspace_bytes(d_in);
}

ONECOMP_API onecomp_status onecomp_hessian_accumulate_ws(const void* X, onecomp_dtype x_dtype, int64_t n_tokens,
                                                         int64_t d_in, int64_t ldx, float* H, void* workspace,
                                                         size_t workspace_bytes, void* hip_stream) {
    const ApiRange range("onecomp_hessian_accumulate_ws");
    if (x_dtype != ONECOMP_F32 && x_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (!H || d_in <= 0 || n_tokens < 0 || ldx < d_in) return ONECOMP_ERR_INVALID_ARG;
    if (d_in % 16 != 0 || d_in > (1 << 20)) return ONECOMP_ERR_INVALID_ARG;
    if (workspace && !aligned(workspace, 256)) return ONECOMP_ERR_WORKSPACE;
    if (n_tokens == 0) return ONECOMP_OK;
    if (!X) return ONECOMP_ERR_INVALID_ARG;
    const size_t esz = (x_dtype == ONECOMP_BF16) ? 2 : 4;
    if (!aligned(X, 16) || (size_t(ldx) * esz) % 16 != 0 || !aligned(H, 16)) return ONECOMP_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (x_dtype == ONECOMP_BF16)
        return gram_accumulate_bf16(X, n_tokens, d_in, ldx, H, workspace, workspace ? workspace_bytes : 0, s);
    return gram_accumulate_f32(X, n_tokens, d_in, ldx, H, s);
}

ONECOMP_API onecomp_status onecomp_accumulate_describe(onecomp_dtype x_dtype, int64_t n_tokens, int64_t d_in, int64_t ldx,
                                                       size_t workspace_bytes, int32_t* out3) {
    if (x_dtype != ONECOMP_F32 && x_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (!out3 || d_in <= 0 || n_tokens < 0 || ldx < d_in) return ONECOMP_ERR_INVALID_ARG;
    if (d_in % 16 != 0 || d_in > (1 << 20)) return ONECOMP_ERR_INVALID_ARG;
    GramPlanInfo info{128, 128, 1};
    const onecomp_status st = x_dtype == ONECOMP_BF16 ? gram_accumulate_bf16(nullptr, n_tokens, d_in, ldx, nullptr, nullptr,
                                                                             workspace_bytes, nullptr, &info)
                                                      : gram_accumulate_f32(nullptr, n_tokens, d_in, ldx, nullptr, nullptr, &info);
    if (st != ONECOMP_OK) return st;
    out3[0] = info.tile_rows;
    out3[1] = info.tile_cols;
    out3[2] = info.launches;
    return ONECOMP_OK;
}

ONECOMP_API onecomp_status onecomp_hessian_accumulate(const void* X, onecomp_dtype x_dtype, int64_t n_tokens, int64_t d_in,
                                          int64_t ldx, float* H, void* hip_stream) {
    return onecomp_hessian_accumulate_ws(X, x_dtype, n_tokens, d_in, ldx, H, nullptr, 0, hip_stream);
}

ONECOMP_API size_t onecomp_factor_workspace_bytes(int64_t d_in) {
    if (d_in <= 0 || d_in % 16 != 0 || d_in > 46336) return 0;
    return factor_workspace_bytes(d_in);
}

ONECOMP_API onecomp_status onecomp_hessian_factor_form(const float* H, int64_t d_in, float damp, int act_order,
                                                       onecomp_factor_form form, int32_t* perm_out, float* F_out,
                                                       int32_t* info, void* workspace, size_t workspace_bytes,
                                                       void* hip_stream) {
    const ApiRange range("onecomp_hessian_factor_form");
    if (form != ONECOMP_FACTOR_INVERSE && form != ONECOMP_FACTOR_BLOCK) return ONECOMP_ERR_UNSUPPORTED;
    if (!H || !F_out || !info || d_in <= 0) return ONECOMP_ERR_INVALID_ARG;
    if (d_in % 16 != 0 || d_in > 46336) return ONECOMP_ERR_INVALID_ARG;
    if (form == ONECOMP_FACTOR_BLOCK && d_in % 128 != 0) return ONECOMP_ERR_UNSUPPORTED;
    if (!(damp >= 0.0f)) return ONECOMP_ERR_INVALID_ARG;
    if (act_order && !perm_out) return ONECOMP_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < factor_workspace_bytes(d_in))
        return ONECOMP_ERR_WORKSPACE;
    return factor_run(H, d_in, damp, act_order, int(form), perm_out, F_out, info, workspace,
                      static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API onecomp_status onecomp_hessian_factor(const float* H, int64_t d_in, float damp, int act_order, int32_t* perm_out,
                                      float* U, int32_t* info, void* workspace, size_t workspace_bytes,
                                      void* hip_stream) {
    return onecomp_hessian_factor_form(H, d_in, damp, act_order, ONECOMP_FACTOR_INVERSE, perm_out, U, info, workspace,
                                       workspace_bytes, hip_stream);
}

ONECOMP_API size_t onecomp_quantize_workspace_bytes(int64_t d_out, int64_t d_in, int block_size) {
    if (d_out <= 0 || d_in <= 0 || block_size != 128 || d_in % 128 != 0) return 0;
    return sweep_workspace_bytes(d_out, d_in, block_size);
}

ONECOMP_API onecomp_status onecomp_quantize_layer_form(const void* W, onecomp_dtype w_dtype, int64_t d_out,
                                                       int64_t d_in, const float* F, onecomp_factor_form form,
                                                       const int32_t* perm, int bits, int group_size, int block_size,
                                                       onecomp_grid grid, uint8_t* Q_codes, float* scales,
                                                       float* zeros, float* W_hat, float* loss, void* workspace,
                                                       size_t workspace_bytes, void* hip_stream) {
    const ApiRange range("onecomp_quantize_layer_form");
    const float* U = F;
    if (w_dtype != ONECOMP_F32 && w_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (grid != ONECOMP_GRID_MINMAX && grid != ONECOMP_GRID_SYMMETRIC && grid != ONECOMP_GRID_MINMAX_MSE &&
        grid != ONECOMP_GRID_SYMMETRIC_MSE)
        return ONECOMP_ERR_UNSUPPORTED;
    if (form != ONECOMP_FACTOR_INVERSE && form != ONECOMP_FACTOR_BLOCK) return ONECOMP_ERR_UNSUPPORTED;
    if (!W || !U || !Q_codes || !scales || !zeros || !loss) return ONECOMP_ERR_INVALID_ARG;
    if (d_out <= 0 || d_in <= 0 || d_out > (1 << 24) || d_in > 65535) return ONECOMP_ERR_INVALID_ARG;
    if (bits != 2 && bits != 3 && bits != 4 && bits != 8) return ONECOMP_ERR_UNSUPPORTED;
    if (block_size != 128) return ONECOMP_ERR_UNSUPPORTED;
    if (group_size <= 0 || d_in % block_size != 0 || d_in % group_size != 0) return ONECOMP_ERR_INVALID_ARG;
    if (group_size % 16 != 0) return ONECOMP_ERR_UNSUPPORTED;
    if (block_size % group_size != 0 && group_size % block_size != 0) return ONECOMP_ERR_INVALID_ARG;
    if (form == ONECOMP_FACTOR_BLOCK && group_size > block_size && group_size != d_in) return ONECOMP_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(U, 16) || !aligned(Q_codes, 4) || (W_hat && !aligned(W_hat, 16)))
        return ONECOMP_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < sweep_workspace_bytes(d_out, d_in, block_size))
        return ONECOMP_ERR_WORKSPACE;
    return sweep_run(W, w_dtype, d_out, d_in, U, int(form), perm, bits, group_size, block_size, int(grid), Q_codes,
                     scales, zeros, W_hat, loss, workspace, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API onecomp_status onecomp_quantize_layer_grid(const void* W, onecomp_dtype w_dtype, int64_t d_out,
                                                       int64_t d_in, const float* U, const int32_t* perm, int bits,
                                                       int group_size, int block_size, onecomp_grid grid,
                                                       uint8_t* Q_codes, float* scales, float* zeros, float* W_hat,
                                                       float* loss, void* workspace, size_t workspace_bytes,
                                                       void* hip_stream) {
    return onecomp_quantize_layer_form(W, w_dtype, d_out, d_in, U, ONECOMP_FACTOR_INVERSE, perm, bits, group_size,
                                       block_size, grid, Q_codes, scales, zeros, W_hat, loss, workspace, workspace_bytes,
                                       hip_stream);
}

ONECOMP_API onecomp_status onecomp_quantize_layer(const void* W, onecomp_dtype w_dtype, int64_t d_out, int64_t d_in,
                                      const float* U, const int32_t* perm, int bits, int group_size, int block_size,
                                      uint8_t* Q_codes, float* scales, float* zeros, float* W_hat, float* loss,
                                      void* workspace, size_t workspace_bytes, void* hip_stream) {
    return onecomp_quantize_layer_grid(W, w_dtype, d_out, d_in, U, perm, bits, group_size, block_size,
                                       ONECOMP_GRID_MINMAX, Q_codes, scales, zeros, W_hat, loss, workspace,
                                       workspace_bytes, hip_stream);
}

ONECOMP_API onecomp_status onecomp_crossgram_accumulate(const void* X_hat, const void* X, onecomp_dtype x_dtype,
                                                        int64_t n_tokens, int64_t d_in, int64_t ldxh, int64_t ldx,
                                                        float* G, void* hip_stream) {
    const ApiRange range("onecomp_crossgram_accumulate");
    if (x_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (!G || d_in <= 0 || n_tokens < 0 || ldxh < d_in || ldx < d_in) return ONECOMP_ERR_INVALID_ARG;
    if (d_in % 16 != 0 || d_in > (1 << 20)) return ONECOMP_ERR_INVALID_ARG;
    if (n_tokens == 0) return ONECOMP_OK;
    if (!X_hat || !X) return ONECOMP_ERR_INVALID_ARG;
    if (!aligned(X_hat, 16) || !aligned(X, 16) || (ldxh * 2) % 16 != 0 || (ldx * 2) % 16 != 0 || !aligned(G, 16))
        return ONECOMP_ERR_INVALID_ARG;
    // the kernel addresses a step of 16 token rows with 32-bit byte offsets
    if (ldxh * 64 >= (int64_t(1) << 31) || ldx * 64 >= (int64_t(1) << 31)) return ONECOMP_ERR_UNSUPPORTED;
    return gram_cross_accumulate_bf16(X_hat, X, n_tokens, d_in, ldxh, ldx, G, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_qep_workspace_bytes(int64_t d_out, int64_t d_in) {
    if (d_out <= 0 || d_in <= 0 || d_in % 16 != 0 || d_in > 65535 || d_out > (1 << 24)) return 0;
    return qep_workspace_bytes(d_out, d_in);
}

ONECOMP_API onecomp_status onecomp_qep_target(const void* W, onecomp_dtype w_dtype, int64_t d_out, int64_t d_in,
                                              const float* G, const float* H, const float* U, const int32_t* perm,
                                              float alpha, float* W_star, void* workspace, size_t workspace_bytes,
                                              void* hip_stream) {
    const ApiRange range("onecomp_qep_target");
    if (w_dtype != ONECOMP_F32 && w_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (!W || !G || !H || !U || !W_star) return ONECOMP_ERR_INVALID_ARG;
    if (d_out <= 0 || d_in <= 0 || d_in % 16 != 0 || d_in > 65535 || d_out > (1 << 24)) return ONECOMP_ERR_INVALID_ARG;
    if (!(alpha >= 0.0f && alpha <= 1.0f)) return ONECOMP_ERR_INVALID_ARG;
    if (static_cast<const void*>(W_star) == W) return ONECOMP_ERR_INVALID_ARG;
    if (!aligned(W, 16) || !aligned(G, 16) || !aligned(H, 16) || !aligned(U, 16) || !aligned(W_star, 16))
        return ONECOMP_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < qep_workspace_bytes(d_out, d_in))
        return ONECOMP_ERR_WORKSPACE;
    return qep_target_run(W, w_dtype, d_out, d_in, G, H, U, perm, alpha, W_star, workspace,
                          static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_jointq_workspace_bytes(int64_t d_out, int64_t d_in, int group_size) {
    if (d_out <= 0 || d_in <= 0 || group_size <= 0 || group_size % 16 != 0 || d_in % group_size != 0) return 0;
    if (group_size > 128 && group_size % 128 != 0) return 0;
    return jointq_workspace_bytes(d_out, d_in, group_size);
}

ONECOMP_API onecomp_status onecomp_jointq_refine(const void* W, onecomp_dtype w_dtype, int64_t d_out, int64_t d_in,
                                                 const float* H, const int32_t* perm, float lam, int bits,
                                                 int group_size,
                                                 onecomp_grid grid, int n_pass, int max_scans, uint8_t* Q_codes,
                                                 float* scales, const float* zeros, float* W_hat, float* objective,
                                                 int32_t* n_moves, void* workspace, size_t workspace_bytes,
                                                 void* hip_stream) {
    const ApiRange range("onecomp_jointq_refine");
    if (w_dtype != ONECOMP_F32 && w_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (grid != ONECOMP_GRID_MINMAX && grid != ONECOMP_GRID_SYMMETRIC && grid != ONECOMP_GRID_MINMAX_MSE &&
        grid != ONECOMP_GRID_SYMMETRIC_MSE)
        return ONECOMP_ERR_UNSUPPORTED;
    if (bits != 2 && bits != 3 && bits != 4 && bits != 8) return ONECOMP_ERR_UNSUPPORTED;
    if (!W || !H || !Q_codes || !scales || !zeros || !objective || !n_moves) return ONECOMP_ERR_INVALID_ARG;
    if (d_out <= 0 || d_in <= 0 || d_out > (1 << 24) || d_in > (1 << 20)) return ONECOMP_ERR_INVALID_ARG;
    if (!(lam >= 0.0f) || n_pass < 0 || max_scans < 1) return ONECOMP_ERR_INVALID_ARG;
    if (group_size <= 0 || d_in % 16 != 0 || d_in % group_size != 0) return ONECOMP_ERR_INVALID_ARG;
    if (group_size % 16 != 0 || (group_size > 128 && group_size % 128 != 0)) return ONECOMP_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(H, 16) || !aligned(Q_codes, 4) || (W_hat && !aligned(W_hat, 16)))
        return ONECOMP_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < jointq_workspace_bytes(d_out, d_in, group_size))
        return ONECOMP_ERR_WORKSPACE;
    return jointq_run(W, w_dtype, d_out, d_in, H, perm, lam, bits, group_size, int(grid), n_pass, max_scans, Q_codes, scales,
                      zeros, W_hat, objective, n_moves, workspace, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_sensitivity_workspace_bytes(void) { return sensitivity_workspace_bytes(); }

ONECOMP_API onecomp_status onecomp_rtn_sensitivity(const void* W, onecomp_dtype w_dtype, int64_t d_out, int64_t d_in,
                                                   const float* a_diag, const float* b_diag, int bits, int group_size,
                                                   onecomp_grid grid, float* err, void* workspace,
                                                   size_t workspace_bytes, void* hip_stream) {
    const ApiRange range("onecomp_rtn_sensitivity");
    if (w_dtype != ONECOMP_F32 && w_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (grid != ONECOMP_GRID_MINMAX && grid != ONECOMP_GRID_SYMMETRIC) return ONECOMP_ERR_UNSUPPORTED;
    if (bits != 2 && bits != 3 && bits != 4 && bits != 8) return ONECOMP_ERR_UNSUPPORTED;
    if (!W || !a_diag || !err) return ONECOMP_ERR_INVALID_ARG;
    if (d_out <= 0 || d_in <= 0 || d_out > (1 << 24) || d_in > (1 << 24)) return ONECOMP_ERR_INVALID_ARG;
    if (group_size <= 0 || d_in % group_size != 0) return ONECOMP_ERR_INVALID_ARG;
    if (group_size % 16 != 0) return ONECOMP_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(a_diag, 16)) return ONECOMP_ERR_INVALID_ARG;   // 16-byte vector loads
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < sensitivity_workspace_bytes())
        return ONECOMP_ERR_WORKSPACE;
    return sensitivity_run(W, w_dtype, d_out, d_in, a_diag, b_diag, bits, group_size, int(grid), err, workspace,
                           static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API onecomp_status onecomp_rtn_sensitivity_static(const void* W, onecomp_dtype w_dtype, int64_t d_out,
                                                          int64_t d_in, const float* a_diag, const float* b_diag,
                                                          int bits, int group_size, onecomp_grid grid, float* err,
                                                          void* hip_stream) {
    const ApiRange range("onecomp_rtn_sensitivity_static");
    if (w_dtype != ONECOMP_F32 && w_dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
    if (grid != ONECOMP_GRID_MINMAX && grid != ONECOMP_GRID_SYMMETRIC) return ONECOMP_ERR_UNSUPPORTED;
    if (bits != 2 && bits != 3 && bits != 4 && bits != 8) return ONECOMP_ERR_UNSUPPORTED;
    if (!W || !a_diag || !err) return ONECOMP_ERR_INVALID_ARG;
    // the built-in scratch holds one partial sum per workgroup of a grid capped at 2048 workgroups, which covers every
    // size up to the limits below; anything beyond them is rejected here, before any launch
    if (d_out <= 0 || d_in <= 0 || d_out > (1 << 24) || d_in > (1 << 24)) return ONECOMP_ERR_INVALID_ARG;
    if (group_size <= 0 || d_in % group_size != 0) return ONECOMP_ERR_INVALID_ARG;
    if (group_size % 16 != 0) return ONECOMP_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(a_diag, 16)) return ONECOMP_ERR_INVALID_ARG;
    return sensitivity_run_static(W, w_dtype, d_out, d_in, a_diag, b_diag, bits, group_size, int(grid), err,
                                  static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API onecomp_status onecomp_mfma_rate_probe(int kind, int waves_per_simd, int random_operands, int64_t iters,
                                                   float* sink, double* flops_out, void* hip_stream) {
    if (kind != 0 && kind != 1) return ONECOMP_ERR_UNSUPPORTED;
    if (waves_per_simd != 1 && waves_per_simd != 2) return ONECOMP_ERR_UNSUPPORTED;
    if (random_operands != 0 && random_operands != 1) return ONECOMP_ERR_INVALID_ARG;
    if (!sink || !flops_out || iters <= 0 || iters > (int64_t(1) << 24)) return ONECOMP_ERR_INVALID_ARG;
    const ApiRange range("onecomp_mfma_rate_probe");
    return mfma_rate_probe(kind, waves_per_simd, random_operands, iters, sink, flops_out,
                           static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_attention_workspace_bytes(const onecomp_attention_shape* shape) {
    if (check_attention(shape) != ONECOMP_OK) return 0;
    return attn::forward_workspace_bytes(shape->dtype, attention_params(shape));
}

ONECOMP_API onecomp_status onecomp_attention_forward(const onecomp_attention_shape* shape, const onecomp_heads* q, const onecomp_heads* k,
                                                     const onecomp_heads* v, const onecomp_heads* out, float* lse, void* workspace,
                                                     size_t workspace_bytes, void* hip_stream) {
    const ApiRange range("onecomp_attention_forward");
    if (const onecomp_status st = check_attention(shape)) return st;
    if (!check_heads(shape, q, shape->total_q) || !check_heads(shape, out, shape->total_q) || !check_heads(shape, k, shape->total_k) ||
        !check_heads(shape, v, shape->total_k) || !aligned(lse, 4))
        return ONECOMP_ERR_INVALID_ARG;
    attn::Params P = attention_params(shape);
    const size_t need = attn::forward_workspace_bytes(shape->dtype, P);
    if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return ONECOMP_ERR_WORKSPACE;
    if (P.total_q == 0) return ONECOMP_OK;
    if (same(out, k, shape->total_k) || same(out, v, shape->total_k)) return ONECOMP_ERR_INVALID_ARG;
    P.q = view(q);
    P.k = view(k);
    P.v = view(v);
    P.o = view(out);
    P.lse = lse;
    P.part = static_cast<float*>(workspace);
    return attn::forward_run(shape->dtype, P, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_attention_backward_workspace_bytes(const onecomp_attention_shape* shape) {
    if (check_attention(shape) != ONECOMP_OK) return 0;
    return attn::backward_workspace_bytes(shape->dtype, attention_params(shape));
}

ONECOMP_API onecomp_status onecomp_attention_backward(const onecomp_attention_shape* shape, const onecomp_heads* q, const onecomp_heads* k,
                                                      const onecomp_heads* v, const onecomp_heads* out, const float* lse,
                                                      const onecomp_heads* d_out, const onecomp_heads* dq, const onecomp_heads* dk,
                                                      const onecomp_heads* dv, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const ApiRange range("onecomp_attention_backward");
    if (const onecomp_status st = check_attention(shape)) return st;
    if (!check_heads(shape, q, shape->total_q) || !check_heads(shape, out, shape->total_q) || !check_heads(shape, d_out, shape->total_q) ||
        !check_heads(shape, dq, shape->total_q) || !check_heads(shape, k, shape->total_k) || !check_heads(shape, v, shape->total_k) ||
        !check_heads(shape, dk, shape->total_k) || !check_heads(shape, dv, shape->total_k) || (!lse && shape->total_q) || !aligned(lse, 4))
        return ONECOMP_ERR_INVALID_ARG;
    attn::Params P = attention_params(shape);
    const size_t need = attn::backward_workspace_bytes(shape->dtype, P);
    if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return ONECOMP_ERR_WORKSPACE;
    // dk and dv are formed from all queries and d_out when dq has been written, dq from all keys and values
    const bool q_k = P.total_q && P.total_k;
    for (const onecomp_heads* in : {q, d_out})
        if (same(dq, in, P.total_q) || same(dk, in, q_k) || same(dv, in, q_k)) return ONECOMP_ERR_INVALID_ARG;
    for (const onecomp_heads* other : {k, v, dk, dv})
        if (same(dq, other, q_k)) return ONECOMP_ERR_INVALID_ARG;
    if (same(dk, dv, P.total_k)) return ONECOMP_ERR_INVALID_ARG;
    P.q = view(q);
    P.k = view(k);
    P.v = view(v);
    P.o = view(out);
    P.d_o = view(d_out);
    P.dq = view(dq);
    P.dk = view(dk);
    P.dv = view(dv);
    P.lse = const_cast<float*>(lse);
    P.aux = static_cast<float*>(workspace);
    return attn::backward_run(shape->dtype, P, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API onecomp_status onecomp_block_norm_forward(const onecomp_norm_shape* shape, const onecomp_rows* h, const onecomp_rows* y,
                                                      const void* weight, const void* bias, const void* post_weight, const void* post_bias,
                                                      const onecomp_rows* gate, const onecomp_rows* h_out, const onecomp_rows* n,
                                                      void* hip_stream) {
    const ApiRange range("onecomp_block_norm_forward");
    if (const onecomp_status st = check_norm(shape)) return st;
    block::Params P;
    if (const onecomp_status st = norm_arguments(shape, P, h, y, weight, bias, post_weight, post_bias, gate)) return st;
    if (!check_rows(shape, h_out) || !check_rows(shape, n) || (!h_out && !n) || (h_out && !y)) return ONECOMP_ERR_INVALID_ARG;
    if (shape->rows == 0) return ONECOMP_OK;
    if (n && (n->data == h->data || (h_out && n->data == h_out->data))) return ONECOMP_ERR_INVALID_ARG;
    if (!apart_or_same(shape, {h_out, n}, {h, y, P.gate_rows ? gate : nullptr})) return ONECOMP_ERR_INVALID_ARG;
    P.h_out = rows_of(h_out);
    P.n = rows_of(n);
    return block::norm_run(shape->dtype, P, false, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_block_norm_workspace_bytes(const onecomp_norm_shape* shape) {
    if (check_norm(shape) != ONECOMP_OK) return 0;
    const bool layer = shape->kind == ONECOMP_NORM_LAYER;
    const int wanted = 1 | (layer ? 2 : 0) | (shape->post_norm ? 4 | (layer ? 8 : 0) : 0) | (shape->gate_kind == ONECOMP_GATE_CHANNEL ? 16 : 0);
    return block::gradient_workspace_bytes(shape->rows, shape->width, wanted);
}

ONECOMP_API onecomp_status onecomp_block_norm_backward(const onecomp_norm_shape* shape, const onecomp_rows* dn, const onecomp_rows* dh_out,
                                                       const onecomp_rows* h, const onecomp_rows* y, const void* weight,
                                                       const void* post_weight, const void* post_bias, const onecomp_rows* gate,
                                                       const onecomp_norm_gradients* out, void* workspace, size_t workspace_bytes,
                                                       void* hip_stream) {
    const ApiRange range("onecomp_block_norm_backward");
    if (const onecomp_status st = check_norm(shape)) return st;
    block::Params P;
    if (const onecomp_status st = norm_arguments(shape, P, h, y, weight, nullptr, post_weight, post_bias, gate)) return st;
    if (!out || (!dn && !dh_out) || !check_rows(shape, dn) || !check_rows(shape, dh_out)) return ONECOMP_ERR_INVALID_ARG;
    if (!check_rows(shape, out->dh) || !check_rows(shape, out->dy) || !check_rows(shape, out->dgate)) return ONECOMP_ERR_INVALID_ARG;
    const bool layer = shape->kind == ONECOMP_NORM_LAYER;
    if ((out->dy && !y) || (out->dgate && shape->gate_kind != ONECOMP_GATE_ROWS) || (out->dgate_channel && shape->gate_kind != ONECOMP_GATE_CHANNEL) ||
        ((out->dweight || out->dbias) && !dn) || ((out->dpost_weight || out->dpost_bias) && !shape->post_norm) || ((out->dbias || out->dpost_bias) && !layer))
        return ONECOMP_ERR_INVALID_ARG;
    void* const params[5] = {out->dweight, out->dbias, out->dpost_weight, out->dpost_bias, out->dgate_channel};
    for (int i = 0; i < 5; ++i) {
        if (!check_param(shape, params[i])) return ONECOMP_ERR_INVALID_ARG;
        P.d_param[i] = params[i];
        P.wanted |= params[i] ? 1 << i : 0;
    }
    if (P.wanted && (!workspace || !aligned(workspace, 256) || workspace_bytes < onecomp_block_norm_workspace_bytes(shape))) return ONECOMP_ERR_WORKSPACE;
    if (shape->rows == 0 && !P.wanted) return ONECOMP_OK;
    if (!apart_or_same(shape, {out->dh, out->dy, out->dgate}, {dn, dh_out, h, y, P.gate_rows ? gate : nullptr})) return ONECOMP_ERR_INVALID_ARG;
    P.part = static_cast<float*>(workspace);
    P.dn = rows_of(dn);
    P.dh_out = rows_of(dh_out);
    P.dh = rows_of(out->dh);
    P.dy = rows_of(out->dy);
    P.dgate = rows_of(out->dgate);
    return block::norm_run(shape->dtype, P, true, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API size_t onecomp_clip_workspace_bytes(void) { return block::clip_workspace_bytes(); }

ONECOMP_API onecomp_status onecomp_clip_gradients(const onecomp_gradient* grads, int n, float max_norm, float* norm, void* workspace,
                                                  size_t workspace_bytes, void* hip_stream) {
    const ApiRange range("onecomp_clip_gradients");
    if (n < 0 || (n > 0 && !grads) || !(max_norm >= 0.f) || !aligned(norm, 4)) return ONECOMP_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const onecomp_gradient& g = grads[i];
        if (g.dtype != ONECOMP_F32 && g.dtype != ONECOMP_BF16) return ONECOMP_ERR_UNSUPPORTED;
        const size_t esz = g.dtype == ONECOMP_BF16 ? 2 : 4;
        if (g.numel < 0 || g.numel > (int64_t(1) << 40) || (g.numel > 0 && (!g.grad || !g.out || !aligned(g.grad, esz) || !aligned(g.out, esz))))
            return ONECOMP_ERR_INVALID_ARG;
    }
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < block::clip_workspace_bytes()) return ONECOMP_ERR_WORKSPACE;
    return block::clip_run(grads, n, max_norm, norm, workspace, static_cast<hipStream_t>(hip_stream));
}

ONECOMP_API const char* onecomp_status_string(onecomp_status status) {
    switch (status) {
        case ONECOMP_OK: return "ok";
        case ONECOMP_ERR_INVALID_ARG: return "invalid argument";
        case ONECOMP_ERR_UNSUPPORTED: return "unsupported dtype, bit width, group size or block size";
        case ONECOMP_ERR_NOT_POSDEF: return "matrix is not positive definite";
        case ONECOMP_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case ONECOMP_ERR_HIP: return "HIP runtime error";
    }
    return "unknown status";
}

ONECOMP_API int onecomp_version(void) { return 200; }

}  // extern "C"
