// Host side of the sequence operators of include/mdlstm.h: argument validation
// (always before the first HIP call), workspace planning and dispatch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "host.hpp"
#include "mdlstm.h"
#include "sequence.hpp"

namespace {

mdlstm_status fail(mdlstm_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return mdl::set_error(st, buf);
}

#define HIP_OR_FAIL(expr)                                                                                   \
    do {                                                                                                    \
        hipError_t _e = (expr);                                                                             \
        if (_e != hipSuccess) return fail(MDLSTM_ERR_DEVICE, "%s: %s", #expr, hipGetErrorString(_e));       \
    } while (0)

#define OK_OR_RETURN(expr)                        \
    do {                                          \
        const mdlstm_status _st = (expr);         \
        if (_st != MDLSTM_OK) return _st;         \
    } while (0)

constexpr int64_t kMaxTokens = (int64_t)1 << 35;  // products with a dimension or a head count stay within int64
constexpr int64_t kMaxStride = (int64_t)1 << 62;

size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }
bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
size_t element(int32_t dtype) { return dtype == MDLSTM_BF16 ? 2 : 4; }

mdlstm_status check_dtype(int32_t dtype) {
    if (dtype != MDLSTM_F32 && dtype != MDLSTM_BF16)
        return fail(MDLSTM_ERR_INVALID_ARG, "dtype %d is not MDLSTM_F32 or MDLSTM_BF16", dtype);
    return MDLSTM_OK;
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
mdlstm_status check_attention(const mdlstm_attention_desc* d) {
    if (!d) return fail(MDLSTM_ERR_INVALID_ARG, "desc is NULL");
    OK_OR_RETURN(check_dtype(d->dtype));
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
        return fail(MDLSTM_ERR_INVALID_ARG, "%d heads are not a multiple of %d key and value heads", d->heads, d->kv_heads);
    if (d->dim_k < 1 || d->dim_v < 1) return fail(MDLSTM_ERR_INVALID_ARG, "dim_k and dim_v must be positive");
    if (d->heads > 1024) return fail(MDLSTM_ERR_UNSUPPORTED, "%d heads: at most 1024", d->heads);
    if (d->dim_k > 128 || d->dim_v > 128)
        return fail(MDLSTM_ERR_UNSUPPORTED, "dim_k %d, dim_v %d: at most 128", d->dim_k, d->dim_v);
    return MDLSTM_OK;
}

mdlstm_status check_sequences(int32_t n, int64_t tokens, int64_t longest) {
    if (n < 0 || n > MDLSTM_MAX_RECTS) return fail(MDLSTM_ERR_INVALID_ARG, "%d examples: 0 to %d", n, MDLSTM_MAX_RECTS);
    if (tokens < 0 || tokens > kMaxTokens || longest < 0 || longest > tokens)
        return fail(MDLSTM_ERR_INVALID_ARG, "%lld tokens, the longest example %lld", (long long)tokens, (long long)longest);
    if (n == 0 && tokens > 0) return fail(MDLSTM_ERR_INVALID_ARG, "%lld tokens of no example", (long long)tokens);
    return MDLSTM_OK;
}

// Strides whose products with `tokens` and `heads` stay within int64, a pointer to whole elements.
mdlstm_status check_view(const mdlstm_heads* v, const char* name, int64_t tokens, int32_t heads, int32_t dtype) {
    if (!v) return fail(MDLSTM_ERR_INVALID_ARG, "%s is NULL", name);
    if (tokens > 0 && !v->d_data) return fail(MDLSTM_ERR_INVALID_ARG, "the device pointer of %s is NULL", name);
    if (misaligned(v->d_data, element(dtype))) return fail(MDLSTM_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (v->token_stride < 0 || v->head_stride < 0)
        return fail(MDLSTM_ERR_INVALID_ARG, "strides %lld, %lld of %s are negative", (long long)v->token_stride,
                    (long long)v->head_stride, name);
    int64_t a, b, c;
    if (__builtin_mul_overflow(v->token_stride, tokens, &a) || __builtin_mul_overflow(v->head_stride, (int64_t)heads, &b) ||
        __builtin_add_overflow(a, b, &c) || c > kMaxStride / 4)
        return fail(MDLSTM_ERR_INVALID_ARG, "strides %lld, %lld of %s are too large", (long long)v->token_stride,
                    (long long)v->head_stride, name);
    return MDLSTM_OK;
}

mdlstm_status check_out(const void* p, const char* name, bool needed, size_t to) {
    if (needed && !p) return fail(MDLSTM_ERR_INVALID_ARG, "%s is NULL", name);
    if (misaligned(p, to)) return fail(MDLSTM_ERR_INVALID_ARG, "%s must be %zu-byte aligned", name, to);
    return MDLSTM_OK;
}

// The bytes of an argument, and whether the call writes them.
struct Span {
    const char* name;
    uintptr_t from, size;
    bool written;
};
Span span(const char* name, const void* p, int64_t bytes, bool written) {
    return Span{name, reinterpret_cast<uintptr_t>(p), p ? (uintptr_t)bytes : 0, written};
}
// From a view's first element to its last.
Span span(const char* name, const mdlstm_heads* v, int64_t tokens, int32_t heads, int32_t dim, int32_t dtype) {
    const int64_t last = (tokens - 1) * v->token_stride + (heads - 1) * v->head_stride + dim;
    return span(name, v->d_data, tokens > 0 ? last * (int64_t)element(dtype) : 0, false);
}

// Nothing that the call writes may overlap anything else: workgroups read and write in no order.
template <size_t N>
mdlstm_status check_apart(const Span (&s)[N]) {
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < N && s[i].written; ++j)
            if (j != i && s[i].size && s[j].size && s[i].from < s[j].from + s[j].size && s[j].from < s[i].from + s[i].size)
                return fail(MDLSTM_ERR_INVALID_ARG, "%s overlaps %s", s[i].name, s[j].name);
    return MDLSTM_OK;
}

mdl::HeadView view(const mdlstm_heads* v, int group, int dim) {
    return mdl::HeadView{v->d_data, v->token_stride, v->head_stride, group, dim};
}

mdl::ScanArgs scan_args(const mdlstm_attention_desc* d, int32_t n, int64_t tokens, int64_t longest,
                        const int64_t* offsets, const int32_t* order, const float* rates) {
    mdl::ScanArgs a{};
    a.n = n;
    a.heads = d->heads;
    a.group = d->heads / d->kv_heads;
    a.dtype = d->dtype;
    a.tokens = tokens;
    a.longest = longest;
    a.offsets = offsets;
    a.order = order;
    a.rates = rates;
    return a;
}

// The roles of a call as far as the workspace depends on them: their dimensions.
void role_dims(mdl::ScanArgs& a, const mdlstm_attention_desc* d, bool backward) {
    a.n_roles = backward ? 3 : 1;
    for (int r = 0; r < a.n_roles; ++r) {
        const bool t = backward && r < 2;  // dq and dk scan the transposed state
        a.role[r].q.dim = a.role[r].k.dim = t ? d->dim_v : d->dim_k;
        a.role[r].v.dim = t ? d->dim_k : d->dim_v;
    }
}

struct AttentionPlan {
    size_t dk, dv, scan, total;
};

AttentionPlan attention_plan(const mdlstm_attention_desc* d, int32_t n, int64_t tokens, int64_t longest, bool backward) {
    AttentionPlan p{};
    size_t off = 0;
    if (backward && d->heads > d->kv_heads) {  // the gradients of shared heads, a share per query head
        p.dk = off;
        off += align_up((size_t)tokens * d->heads * d->dim_k * 4);
        p.dv = off;
        off += align_up((size_t)tokens * d->heads * d->dim_v * 4);
    }
    p.scan = off;
    mdl::ScanArgs a = scan_args(d, n, tokens, longest, nullptr, nullptr, nullptr);
    role_dims(a, d, backward);
    off += align_up(mdl::scan_workspace_bytes(a));
    p.total = off;
    return p;
}

mdlstm_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws || have < need) return fail(MDLSTM_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : 0, need);
    if (misaligned(ws, 16)) return fail(MDLSTM_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    return MDLSTM_OK;
}

// ---------------------------------------------------------------------------
// Norm and dropout
// ---------------------------------------------------------------------------
mdlstm_status check_p(double p) {
    if (!(p >= 0.0 && p <= 1.0)) return fail(MDLSTM_ERR_INVALID_ARG, "dropout probability %g is not in [0, 1]", p);
    return MDLSTM_OK;
}

mdl::Drop drop_of(double p, uint64_t seed, uint64_t call) {
    mdl::Drop d{seed, call, (uint32_t)std::nearbyint(p * 65536.0), 0.0f};
    d.scale = d.threshold < 65536 ? (float)(65536.0 / (65536 - d.threshold)) : 0.0f;
    return d;
}

mdlstm_status check_rows(const void* p, const char* name, int64_t rows, int64_t cols, int64_t stride, int32_t dtype) {
    if (rows > 0 && cols > 0 && !p) return fail(MDLSTM_ERR_INVALID_ARG, "%s is NULL", name);
    if (misaligned(p, element(dtype))) return fail(MDLSTM_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    int64_t a;
    if (stride < cols || __builtin_mul_overflow(stride, rows, &a) || a > kMaxStride / 4)
        return fail(MDLSTM_ERR_INVALID_ARG, "rows of %s are %lld elements apart, %lld long", name, (long long)stride,
                    (long long)cols);
    return MDLSTM_OK;
}

mdlstm_status check_norm(const mdlstm_norm_desc* d, int64_t rows) {
    if (!d) return fail(MDLSTM_ERR_INVALID_ARG, "desc is NULL");
    OK_OR_RETURN(check_dtype(d->dtype));
    if (d->cols < 1) return fail(MDLSTM_ERR_INVALID_ARG, "cols %d must be positive", d->cols);
    if (d->cols > mdl::MAX_NORM_COLS) return fail(MDLSTM_ERR_UNSUPPORTED, "cols %d: at most %d", d->cols, mdl::MAX_NORM_COLS);
    if (!(d->eps > 0.0f) || std::isinf(d->eps)) return fail(MDLSTM_ERR_INVALID_ARG, "eps %g must be positive", d->eps);
    OK_OR_RETURN(check_p(d->p));
    if (rows < 0 || rows > 0x7fffffff) return fail(MDLSTM_ERR_INVALID_ARG, "%lld rows: 0 to 2^31 - 1", (long long)rows);
    return MDLSTM_OK;
}

size_t norm_workspace(const mdlstm_norm_desc* d, int64_t rows) {
    return align_up((size_t)mdl::norm_bwd_groups(d->cols, d->dtype, rows) * d->cols * 4 + 16);
}

}  // namespace

extern "C" {

size_t mdlstm_attention_workspace_bytes(const mdlstm_attention_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                        int32_t backward) {
    if (check_attention(desc) != MDLSTM_OK || check_sequences(n, tokens, longest) != MDLSTM_OK) return 0;
    return attention_plan(desc, n, tokens, longest, backward != 0).total;
}

mdlstm_status mdlstm_attention_forward(const mdlstm_attention_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                       const int64_t* d_offsets, const int32_t* d_order, const float* d_rates,
                                       const mdlstm_heads* q,
                                       const mdlstm_heads* k, const mdlstm_heads* v, const float* d_state, void* d_o,
                                       float* d_final, void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_attention(desc));
    OK_OR_RETURN(check_sequences(n, tokens, longest));
    const int group = desc->heads / desc->kv_heads;
    OK_OR_RETURN(check_view(q, "q", tokens, desc->heads, desc->dtype));
    OK_OR_RETURN(check_view(k, "k", tokens, desc->kv_heads, desc->dtype));
    OK_OR_RETURN(check_view(v, "v", tokens, desc->kv_heads, desc->dtype));
    OK_OR_RETURN(check_out(d_offsets, "offsets", n > 0, 8));
    OK_OR_RETURN(check_out(d_order, "order", false, 4));
    OK_OR_RETURN(check_out(d_rates, "rates", n > 0, 4));
    OK_OR_RETURN(check_out(d_state, "state", false, 16));
    OK_OR_RETURN(check_out(d_o, "o", tokens > 0, 16));
    OK_OR_RETURN(check_out(d_final, "final", false, 16));
    const AttentionPlan p = attention_plan(desc, n, tokens, longest, false);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, p.total));
    const int64_t es = (int64_t)element(desc->dtype), states = (int64_t)n * desc->heads * desc->dim_k * desc->dim_v * 4;
    OK_OR_RETURN(check_apart({span("o", d_o, tokens * desc->heads * desc->dim_v * es, true), span("final", d_final, states, true),
                              span("the workspace", d_workspace, (int64_t)p.total, true),
                              span("q", q, tokens, desc->heads, desc->dim_k, desc->dtype),
                              span("k", k, tokens, desc->kv_heads, desc->dim_k, desc->dtype),
                              span("v", v, tokens, desc->kv_heads, desc->dim_v, desc->dtype), span("state", d_state, states, false),
                              span("offsets", d_offsets, ((int64_t)n + 1) * 8, false), span("order", d_order, (int64_t)n * 4, false),
                              span("rates", d_rates, (int64_t)desc->heads * 4, false)}));
    if (n == 0) return MDLSTM_OK;
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, p.total, stream));
    mdl::ScanArgs a = scan_args(desc, n, tokens, longest, d_offsets, d_order, d_rates);
    a.n_roles = 1;
    a.ws = static_cast<char*>(d_workspace) + p.scan;
    a.role[0] = mdl::ScanRole{view(q, 1, desc->dim_k), view(k, group, desc->dim_k), view(v, group, desc->dim_v),
                              d_o, d_state, d_final, desc->scale, 1.0f, 0, 0, 0};
    HIP_OR_FAIL(mdl::launch_scan(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_attention_backward(const mdlstm_attention_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                        const int64_t* d_offsets, const int32_t* d_order, const float* d_rates,
                                       const mdlstm_heads* q,
                                        const mdlstm_heads* k, const mdlstm_heads* v, const float* d_state,
                                        const mdlstm_heads* grad_o, const float* d_dfinal, void* d_dq, void* d_dk,
                                        void* d_dv, float* d_dstate, void* d_workspace, size_t workspace_bytes,
                                        void* stream) {
    OK_OR_RETURN(check_attention(desc));
    OK_OR_RETURN(check_sequences(n, tokens, longest));
    const int group = desc->heads / desc->kv_heads;
    OK_OR_RETURN(check_view(q, "q", tokens, desc->heads, desc->dtype));
    OK_OR_RETURN(check_view(k, "k", tokens, desc->kv_heads, desc->dtype));
    OK_OR_RETURN(check_view(v, "v", tokens, desc->kv_heads, desc->dtype));
    OK_OR_RETURN(check_view(grad_o, "grad_o", tokens, desc->heads, desc->dtype));
    OK_OR_RETURN(check_out(d_offsets, "offsets", n > 0, 8));
    OK_OR_RETURN(check_out(d_order, "order", false, 4));
    OK_OR_RETURN(check_out(d_rates, "rates", n > 0, 4));
    OK_OR_RETURN(check_out(d_state, "state", false, 16));
    OK_OR_RETURN(check_out(d_dfinal, "dfinal", false, 16));
    OK_OR_RETURN(check_out(d_dq, "dq", tokens > 0, 16));
    OK_OR_RETURN(check_out(d_dk, "dk", tokens > 0, 16));
    OK_OR_RETURN(check_out(d_dv, "dv", tokens > 0, 16));
    OK_OR_RETURN(check_out(d_dstate, "dstate", false, 16));
    const AttentionPlan p = attention_plan(desc, n, tokens, longest, true);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, p.total));
    const int64_t es = (int64_t)element(desc->dtype), states = (int64_t)n * desc->heads * desc->dim_k * desc->dim_v * 4;
    OK_OR_RETURN(check_apart({span("dq", d_dq, tokens * desc->heads * desc->dim_k * es, true),
                              span("dk", d_dk, tokens * desc->kv_heads * desc->dim_k * es, true),
                              span("dv", d_dv, tokens * desc->kv_heads * desc->dim_v * es, true),
                              span("dstate", d_dstate, states, true), span("the workspace", d_workspace, (int64_t)p.total, true),
                              span("q", q, tokens, desc->heads, desc->dim_k, desc->dtype),
                              span("k", k, tokens, desc->kv_heads, desc->dim_k, desc->dtype),
                              span("v", v, tokens, desc->kv_heads, desc->dim_v, desc->dtype), span("state", d_state, states, false),
                              span("grad_o", grad_o, tokens, desc->heads, desc->dim_v, desc->dtype),
                              span("dfinal", d_dfinal, states, false), span("offsets", d_offsets, ((int64_t)n + 1) * 8, false),
                              span("order", d_order, (int64_t)n * 4, false),
                              span("rates", d_rates, (int64_t)desc->heads * 4, false)}));
    if (n == 0) return MDLSTM_OK;
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, p.total, stream));
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(d_workspace);
    const mdl::HeadView qv = view(q, 1, desc->dim_k), kv = view(k, group, desc->dim_k), vv = view(v, group, desc->dim_v),
                        gv = view(grad_o, 1, desc->dim_v);
    const int shared = group > 1;
    void* dk = shared ? ws + p.dk : d_dk;
    void* dv = shared ? ws + p.dv : d_dv;
    mdl::ScanArgs a = scan_args(desc, n, tokens, longest, d_offsets, d_order, d_rates);
    a.n_roles = 3;
    a.ws = ws + p.scan;
    a.role[0] = mdl::ScanRole{gv, vv, kv, d_dq, d_state, nullptr, desc->scale, 1.0f, 0, 1, 0};
    a.role[1] = mdl::ScanRole{vv, gv, qv, dk, d_dfinal, nullptr, 1.0f, desc->scale, 1, 1, shared};
    a.role[2] = mdl::ScanRole{kv, qv, gv, dv, d_dfinal, d_dstate, 1.0f, desc->scale, 1, 0, shared};
    HIP_OR_FAIL(mdl::launch_scan(a, s));
    if (shared && tokens > 0) {
        HIP_OR_FAIL(mdl::launch_sum_heads(tokens, desc->kv_heads, group, desc->dim_k, desc->dtype,
                                          static_cast<const float*>(dk), d_dk, s));
        HIP_OR_FAIL(mdl::launch_sum_heads(tokens, desc->kv_heads, group, desc->dim_v, desc->dtype,
                                          static_cast<const float*>(dv), d_dv, s));
    }
    return MDLSTM_OK;
}

mdlstm_status mdlstm_attention_step(const mdlstm_attention_desc* desc, int32_t n, const float* d_rates,
                                    const mdlstm_heads* q, const mdlstm_heads* k, const mdlstm_heads* v,
                                    float* d_state, int64_t slots, const int32_t* d_slots, void* d_o, void* stream) {
    OK_OR_RETURN(check_attention(desc));
    OK_OR_RETURN(check_sequences(n, n, n));
    if (slots < 0 || slots > kMaxTokens) return fail(MDLSTM_ERR_INVALID_ARG, "%lld slots", (long long)slots);
    if (!d_slots && n > slots) return fail(MDLSTM_ERR_INVALID_ARG, "%d rows for %lld slots", n, (long long)slots);
    const int group = desc->heads / desc->kv_heads;
    OK_OR_RETURN(check_view(q, "q", n, desc->heads, desc->dtype));
    OK_OR_RETURN(check_view(k, "k", n, desc->kv_heads, desc->dtype));
    OK_OR_RETURN(check_view(v, "v", n, desc->kv_heads, desc->dtype));
    OK_OR_RETURN(check_out(d_rates, "rates", n > 0, 4));
    OK_OR_RETURN(check_out(d_state, "state", n > 0 && slots > 0, 16));
    OK_OR_RETURN(check_out(d_slots, "slots", false, 4));
    OK_OR_RETURN(check_out(d_o, "o", n > 0, 16));
    if (n == 0) return MDLSTM_OK;
    mdl::StepArgs a{};
    a.n = n;
    a.heads = desc->heads;
    a.dtype = desc->dtype;
    a.q = view(q, 1, desc->dim_k);
    a.k = view(k, group, desc->dim_k);
    a.v = view(v, group, desc->dim_v);
    a.rates = d_rates;
    a.state = d_state;
    a.slots = slots;
    a.slot = d_slots;
    a.out = d_o;
    a.scale = desc->scale;
    HIP_OR_FAIL(mdl::launch_step(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_dropout(int32_t dtype, int64_t rows, int64_t cols, const void* d_x, int64_t x_stride, double p,
                             uint64_t seed, uint64_t call, const void* d_residual, int64_t residual_stride, void* d_y,
                             void* stream) {
    OK_OR_RETURN(check_dtype(dtype));
    OK_OR_RETURN(check_p(p));
    int64_t total;
    if (rows < 0 || cols < 0 || __builtin_mul_overflow(rows, cols, &total) || total > kMaxTokens)
        return fail(MDLSTM_ERR_INVALID_ARG, "%lld rows of %lld elements", (long long)rows, (long long)cols);
    OK_OR_RETURN(check_rows(d_x, "x", rows, cols, x_stride, dtype));
    if (d_residual) OK_OR_RETURN(check_rows(d_residual, "residual", rows, cols, residual_stride, dtype));
    OK_OR_RETURN(check_rows(d_y, "y", rows, cols, cols, dtype));
    if (total == 0) return MDLSTM_OK;
    mdl::DropoutArgs a{dtype, rows, cols, x_stride, residual_stride, d_x, d_residual, d_y, drop_of(p, seed, call)};
    HIP_OR_FAIL(mdl::launch_dropout(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_norm_forward(const mdlstm_norm_desc* desc, int64_t rows, const void* d_x, int64_t x_stride,
                                  const void* d_residual, int64_t residual_stride, const float* d_w, uint64_t seed,
                                  uint64_t call, void* d_h, void* d_y, uint8_t* d_y8, float* d_scale, float* d_rstd,
                                  void* stream) {
    OK_OR_RETURN(check_norm(desc, rows));
    const int64_t cols = desc->cols;
    OK_OR_RETURN(check_rows(d_x, "x", rows, cols, x_stride, desc->dtype));
    if (d_residual) OK_OR_RETURN(check_rows(d_residual, "residual", rows, cols, residual_stride, desc->dtype));
    if (rows > 0 && (!d_y) == (!d_y8)) return fail(MDLSTM_ERR_INVALID_ARG, "one of y and y8 must be given");
    if (rows > 0 && (!d_y8) != (!d_scale)) return fail(MDLSTM_ERR_INVALID_ARG, "y8 and scale go together");
    const mdl::Drop drop = drop_of(desc->p, seed, call);
    if (rows > 0 && !d_h && (d_residual || drop.threshold))
        return fail(MDLSTM_ERR_INVALID_ARG, "h is NULL with a residual or dropout");
    OK_OR_RETURN(check_out(d_h, "h", false, element(desc->dtype)));
    OK_OR_RETURN(check_out(d_y, "y", false, element(desc->dtype)));
    OK_OR_RETURN(check_out(d_w, "w", rows > 0, 4));
    OK_OR_RETURN(check_out(d_scale, "scale", false, 4));
    OK_OR_RETURN(check_out(d_rstd, "rstd", false, 4));
    if (rows == 0) return MDLSTM_OK;
    mdl::NormArgs a{};
    a.cols = desc->cols;
    a.dtype = desc->dtype;
    a.rows = rows;
    a.eps = desc->eps;
    a.drop = drop;
    a.w = d_w;
    a.x = d_x;
    a.x_stride = x_stride;
    a.residual = d_residual;
    a.r_stride = residual_stride;
    a.h = d_h;
    a.y = d_y;
    a.y8 = d_y8;
    a.scale = d_scale;
    a.rstd = d_rstd;
    HIP_OR_FAIL(mdl::launch_norm_fwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

size_t mdlstm_norm_workspace_bytes(const mdlstm_norm_desc* desc, int64_t rows) {
    if (check_norm(desc, rows) != MDLSTM_OK) return 0;
    return norm_workspace(desc, rows);
}

mdlstm_status mdlstm_norm_backward(const mdlstm_norm_desc* desc, int64_t rows, const void* d_h, int64_t h_stride,
                                   const float* d_rstd, const float* d_w, const void* d_dy, const void* d_dh,
                                   uint64_t seed, uint64_t call, void* d_dx, void* d_dresidual, float* d_dw,
                                   void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_norm(desc, rows));
    const int64_t cols = desc->cols;
    OK_OR_RETURN(check_rows(d_h, "h", rows, cols, h_stride, desc->dtype));
    OK_OR_RETURN(check_rows(d_dy, "dy", rows, cols, cols, desc->dtype));
    OK_OR_RETURN(check_rows(d_dx, "dx", rows, cols, cols, desc->dtype));
    OK_OR_RETURN(check_out(d_dh, "dh", false, element(desc->dtype)));
    OK_OR_RETURN(check_out(d_dresidual, "dresidual", false, element(desc->dtype)));
    OK_OR_RETURN(check_out(d_rstd, "rstd", rows > 0, 4));
    OK_OR_RETURN(check_out(d_w, "w", true, 4));
    OK_OR_RETURN(check_out(d_dw, "dw", true, 4));
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, norm_workspace(desc, rows)));
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, norm_workspace(desc, rows), stream));
    mdl::NormArgs a{};
    a.cols = desc->cols;
    a.dtype = desc->dtype;
    a.rows = rows;
    a.eps = desc->eps;
    a.drop = drop_of(desc->p, seed, call);
    a.w = d_w;
    a.rstd = const_cast<float*>(d_rstd);
    a.hin = d_h;
    a.h_stride = h_stride;
    a.dy = d_dy;
    a.dh = d_dh;
    a.dx = d_dx;
    a.dres = d_dresidual;
    a.part = static_cast<float*>(d_workspace);
    a.dw = d_dw;
    HIP_OR_FAIL(mdl::launch_norm_bwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

}  // extern "C"
