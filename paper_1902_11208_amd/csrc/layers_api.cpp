// Host side of the gated recurrence, the group norm and the loss over a vocabulary
// of include/mdlstm.h: argument validation (always before the first HIP call), workspace planning and
// dispatch.
#include <algorithm>
#include <cmath>

#include "checks.hpp"
#include "groupnorm.hpp"
#include "recurrence.hpp"
#include "vocabulary.hpp"

namespace {

constexpr int32_t kMaxChannels = 1 << 20;

mdl::Packed packed(int32_t n, int64_t tokens, int64_t longest, const int64_t* offsets, const int32_t* order) {
    return mdl::Packed{n, tokens, longest, offsets, order, 0, 0};
}

// From the first row's first element to the last row's last.
int64_t rows_bytes(int64_t rows, int64_t cols, int64_t stride, int32_t dtype) {
    return rows > 0 ? ((rows - 1) * stride + cols) * (int64_t)element(dtype) : 0;
}

mdlstm_status check_recurrence(const mdlstm_recurrence_desc* d) {
    if (!d) return fail(MDLSTM_ERR_INVALID_ARG, "desc is NULL");
    OK_OR_RETURN(check_dtype(d->dtype));
    if (d->channels < 1) return fail(MDLSTM_ERR_INVALID_ARG, "%d channels must be positive", d->channels);
    if (d->channels > kMaxChannels) return fail(MDLSTM_ERR_UNSUPPORTED, "%d channels: at most %d", d->channels, kMaxChannels);
    if (d->gate != MDLSTM_GATE_NONE && d->gate != MDLSTM_GATE_SIGMOID)
        return fail(MDLSTM_ERR_INVALID_ARG, "gate %d is not MDLSTM_GATE_NONE or MDLSTM_GATE_SIGMOID", d->gate);
    return MDLSTM_OK;
}

// Rows whose distance within a workgroup's tokens (128 in the recurrence, up to 512 between
// a thread's in the group norm) stays within 32 bits of bytes.
mdlstm_status check_token_rows(const void* p, const char* name, int64_t tokens, int64_t cols, int64_t stride, int32_t dtype) {
    OK_OR_RETURN(check_rows(p, name, tokens, cols, stride, dtype));
    if (tokens > 1 && stride > kMaxChannels)
        return fail(MDLSTM_ERR_UNSUPPORTED, "rows of %s are %lld elements apart: at most %d", name, (long long)stride, kMaxChannels);
    return MDLSTM_OK;
}

mdl::RecurrenceArgs recurrence_args(const mdlstm_recurrence_desc* d, const mdl::Packed& seqs) {
    mdl::RecurrenceArgs a{};
    a.seqs = seqs;
    a.channels = d->channels;
    a.dtype = d->dtype;
    a.sigmoid = d->gate == MDLSTM_GATE_SIGMOID;
    return a;
}

int64_t marks_bytes(const mdlstm_recurrence_desc* d, int64_t tokens) {
    return (tokens / mdl::kRecurrenceTile + 1) * d->channels * 4;
}

mdlstm_status check_group_norm(const mdlstm_group_norm_desc* d) {
    if (!d) return fail(MDLSTM_ERR_INVALID_ARG, "desc is NULL");
    OK_OR_RETURN(check_dtype(d->dtype));
    if (d->channels < 1 || d->groups < 1 || d->channels % d->groups)
        return fail(MDLSTM_ERR_INVALID_ARG, "%d channels are not a multiple of %d groups", d->channels, d->groups);
    if (d->channels > kMaxChannels) return fail(MDLSTM_ERR_UNSUPPORTED, "%d channels: at most %d", d->channels, kMaxChannels);
    if (d->channels / d->groups > mdl::kMaxGroupChannels)
        return fail(MDLSTM_ERR_UNSUPPORTED, "%d channels in a group: at most %d", d->channels / d->groups, mdl::kMaxGroupChannels);
    if (d->activation < MDLSTM_NO_ACTIVATION || d->activation > MDLSTM_SILU)
        return fail(MDLSTM_ERR_INVALID_ARG, "activation %d is not a mdlstm_activation", d->activation);
    if (!(d->eps > 0.0f) || std::isinf(d->eps)) return fail(MDLSTM_ERR_INVALID_ARG, "eps %g must be positive", d->eps);
    return MDLSTM_OK;
}

mdl::GroupNormArgs group_norm_args(const mdlstm_group_norm_desc* d, const mdl::Packed& seqs) {
    mdl::GroupNormArgs a{};
    a.seqs = seqs;
    a.channels = d->channels;
    a.groups = d->groups;
    a.dtype = d->dtype;
    a.act = d->activation;
    a.eps = d->eps;
    return a;
}

mdlstm_status check_vocabulary(const mdlstm_vocabulary_desc* d, int64_t rows) {
    if (!d) return fail(MDLSTM_ERR_INVALID_ARG, "desc is NULL");
    OK_OR_RETURN(check_dtype(d->dtype));
    if (d->dim < 1 || d->vocab < 1) return fail(MDLSTM_ERR_INVALID_ARG, "dim %d and vocab %d must be positive", d->dim, d->vocab);
    if (d->dim > mdl::kMaxVocabularyDim || d->vocab > mdl::kMaxVocabulary)
        return fail(MDLSTM_ERR_UNSUPPORTED, "dim %d, vocab %d: at most %d and %d", d->dim, d->vocab, mdl::kMaxVocabularyDim,
                    mdl::kMaxVocabulary);
    if (rows < 0) return fail(MDLSTM_ERR_INVALID_ARG, "%lld rows", (long long)rows);
    if (rows > mdl::kMaxVocabularyRows)
        return fail(MDLSTM_ERR_UNSUPPORTED, "%lld rows: at most %lld", (long long)rows, (long long)mdl::kMaxVocabularyRows);
    return MDLSTM_OK;
}

mdl::VocabularyArgs vocabulary_args(const mdlstm_vocabulary_desc* d, int64_t rows) {
    mdl::VocabularyArgs a{};
    a.dtype = d->dtype;
    a.dim = d->dim;
    a.vocab = d->vocab;
    a.rows = rows;
    return a;
}

}  // namespace

extern "C" {

size_t mdlstm_recurrence_workspace_bytes(const mdlstm_recurrence_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                         int32_t) {  // both directions cut the same segments
    if (check_recurrence(desc) != MDLSTM_OK || check_sequences(n, tokens, longest) != MDLSTM_OK) return 0;
    return mdl::recurrence_workspace_bytes(recurrence_args(desc, packed(n, tokens, longest, nullptr, nullptr)));
}

size_t mdlstm_recurrence_marks_bytes(const mdlstm_recurrence_desc* desc, int64_t tokens) {
    if (check_recurrence(desc) != MDLSTM_OK || check_sequences(1, tokens, tokens) != MDLSTM_OK) return 0;
    return (size_t)std::max<int64_t>(marks_bytes(desc, tokens), 16);
}

mdlstm_status mdlstm_recurrence_forward(const mdlstm_recurrence_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                        const int64_t* d_offsets, const int32_t* d_order, const void* d_z, int64_t z_stride,
                                        const void* d_x, int64_t x_stride, const float* d_state, void* d_h, float* d_final,
                                        float* d_marks, void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_recurrence(desc));
    OK_OR_RETURN(check_sequences(n, tokens, longest));
    const int64_t cols = desc->channels, es = (int64_t)element(desc->dtype);
    OK_OR_RETURN(check_token_rows(d_z, "z", tokens, cols, z_stride, desc->dtype));
    OK_OR_RETURN(check_token_rows(d_x, "x", tokens, cols, x_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_offsets, "offsets", n > 0, 8));
    OK_OR_RETURN(check_out(d_order, "order", false, 4));
    OK_OR_RETURN(check_out(d_state, "state", false, 4));
    OK_OR_RETURN(check_out(d_h, "h", tokens > 0, es));
    OK_OR_RETURN(check_out(d_final, "final", false, 4));
    OK_OR_RETURN(check_out(d_marks, "marks", false, 4));
    mdl::RecurrenceArgs a = recurrence_args(desc, packed(n, tokens, longest, d_offsets, d_order));
    const size_t need = mdl::recurrence_workspace_bytes(a);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, need));
    OK_OR_RETURN(check_apart({span("h", d_h, tokens * cols * es, true), span("final", d_final, n * cols * 4, true),
                              span("marks", d_marks, marks_bytes(desc, tokens), true),
                              span("the workspace", d_workspace, (int64_t)need, true),
                              span("z", d_z, rows_bytes(tokens, cols, z_stride, desc->dtype), false),
                              span("x", d_x, rows_bytes(tokens, cols, x_stride, desc->dtype), false),
                              span("state", d_state, n * cols * 4, false), span("offsets", d_offsets, ((int64_t)n + 1) * 8, false),
                              span("order", d_order, (int64_t)n * 4, false)}));
    if (n == 0) return MDLSTM_OK;
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, need, stream));
    a.z = mdl::RowView{d_z, z_stride};
    a.x = mdl::RowView{d_x, x_stride};
    a.state = d_state;
    a.marks = d_marks;
    a.h = d_h;
    a.final_state = d_final;
    a.ws = d_workspace;
    HIP_OR_FAIL(mdl::launch_recurrence_fwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_recurrence_backward(const mdlstm_recurrence_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                         const int64_t* d_offsets, const int32_t* d_order, const void* d_z, int64_t z_stride,
                                         const void* d_x, int64_t x_stride, const float* d_state, const float* d_marks,
                                         const void* d_dh, int64_t dh_stride, const float* d_dfinal, void* d_dz, void* d_dx,
                                         float* d_dstate, void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_recurrence(desc));
    OK_OR_RETURN(check_sequences(n, tokens, longest));
    const int64_t cols = desc->channels, es = (int64_t)element(desc->dtype);
    OK_OR_RETURN(check_token_rows(d_z, "z", tokens, cols, z_stride, desc->dtype));
    OK_OR_RETURN(check_token_rows(d_x, "x", tokens, cols, x_stride, desc->dtype));
    OK_OR_RETURN(check_token_rows(d_dh, "dh", tokens, cols, dh_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_offsets, "offsets", n > 0, 8));
    OK_OR_RETURN(check_out(d_order, "order", false, 4));
    OK_OR_RETURN(check_out(d_state, "state", false, 4));
    OK_OR_RETURN(check_out(d_marks, "marks", tokens > 0, 4));
    OK_OR_RETURN(check_out(d_dfinal, "dfinal", false, 4));
    OK_OR_RETURN(check_out(d_dz, "dz", tokens > 0, es));
    OK_OR_RETURN(check_out(d_dx, "dx", tokens > 0, es));
    OK_OR_RETURN(check_out(d_dstate, "dstate", false, 4));
    mdl::RecurrenceArgs a = recurrence_args(desc, packed(n, tokens, longest, d_offsets, d_order));
    const size_t need = mdl::recurrence_workspace_bytes(a);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, need));
    OK_OR_RETURN(check_apart({span("dz", d_dz, tokens * cols * es, true), span("dx", d_dx, tokens * cols * es, true),
                              span("dstate", d_dstate, n * cols * 4, true), span("the workspace", d_workspace, (int64_t)need, true),
                              span("z", d_z, rows_bytes(tokens, cols, z_stride, desc->dtype), false),
                              span("x", d_x, rows_bytes(tokens, cols, x_stride, desc->dtype), false),
                              span("dh", d_dh, rows_bytes(tokens, cols, dh_stride, desc->dtype), false),
                              span("state", d_state, n * cols * 4, false), span("marks", d_marks, marks_bytes(desc, tokens), false),
                              span("dfinal", d_dfinal, n * cols * 4, false), span("offsets", d_offsets, ((int64_t)n + 1) * 8, false),
                              span("order", d_order, (int64_t)n * 4, false)}));
    if (n == 0) return MDLSTM_OK;
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, need, stream));
    a.z = mdl::RowView{d_z, z_stride};
    a.x = mdl::RowView{d_x, x_stride};
    a.dh = mdl::RowView{d_dh, dh_stride};
    a.state = d_state;
    a.marks = const_cast<float*>(d_marks);
    a.dfinal = d_dfinal;
    a.dz = d_dz;
    a.dx = d_dx;
    a.dstate = d_dstate;
    a.ws = d_workspace;
    HIP_OR_FAIL(mdl::launch_recurrence_bwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_recurrence_step(const mdlstm_recurrence_desc* desc, int32_t n, const void* d_z, int64_t z_stride,
                                     const void* d_x, int64_t x_stride, float* d_state, int64_t slots,
                                     const int32_t* d_slots, void* d_h, void* stream) {
    OK_OR_RETURN(check_recurrence(desc));
    OK_OR_RETURN(check_sequences(n, n, n));
    if (slots < 0 || slots > kMaxTokens) return fail(MDLSTM_ERR_INVALID_ARG, "%lld slots", (long long)slots);
    if (!d_slots && n > slots) return fail(MDLSTM_ERR_INVALID_ARG, "%d rows for %lld slots", n, (long long)slots);
    const int64_t cols = desc->channels, es = (int64_t)element(desc->dtype);
    OK_OR_RETURN(check_rows(d_z, "z", n, cols, z_stride, desc->dtype));
    OK_OR_RETURN(check_rows(d_x, "x", n, cols, x_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_state, "state", n > 0 && slots > 0, 4));
    OK_OR_RETURN(check_out(d_slots, "slots", false, 4));
    OK_OR_RETURN(check_out(d_h, "h", n > 0, es));
    OK_OR_RETURN(check_apart({span("h", d_h, n * cols * es, true), span("state", d_state, slots * cols * 4, true),
                              span("z", d_z, rows_bytes(n, cols, z_stride, desc->dtype), false),
                              span("x", d_x, rows_bytes(n, cols, x_stride, desc->dtype), false),
                              span("slots", d_slots, (int64_t)n * 4, false)}));
    if (n == 0) return MDLSTM_OK;
    const mdl::AdvanceArgs a{n, desc->channels, desc->dtype, desc->gate == MDLSTM_GATE_SIGMOID, mdl::RowView{d_z, z_stride},
                             mdl::RowView{d_x, x_stride}, d_state, slots, d_slots, d_h};
    HIP_OR_FAIL(mdl::launch_advance(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

size_t mdlstm_group_norm_workspace_bytes(const mdlstm_group_norm_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                         int32_t backward) {
    if (check_group_norm(desc) != MDLSTM_OK || check_sequences(n, tokens, longest) != MDLSTM_OK) return 0;
    return mdl::groupnorm_workspace_bytes(group_norm_args(desc, packed(n, tokens, longest, nullptr, nullptr)), backward != 0);
}

mdlstm_status mdlstm_group_norm_forward(const mdlstm_group_norm_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                        const int64_t* d_offsets, const int32_t* d_order, const void* d_x, int64_t x_stride,
                                        const float* d_w, const float* d_b, void* d_y, float* d_mean, float* d_rstd,
                                        void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_group_norm(desc));
    OK_OR_RETURN(check_sequences(n, tokens, longest));
    const int64_t cols = desc->channels, es = (int64_t)element(desc->dtype), stats = (int64_t)n * desc->groups * 4;
    OK_OR_RETURN(check_token_rows(d_x, "x", tokens, cols, x_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_offsets, "offsets", n > 0, 8));
    OK_OR_RETURN(check_out(d_order, "order", false, 4));
    OK_OR_RETURN(check_out(d_w, "w", n > 0, 4));
    OK_OR_RETURN(check_out(d_b, "b", n > 0, 4));
    OK_OR_RETURN(check_out(d_y, "y", tokens > 0, es));
    OK_OR_RETURN(check_out(d_mean, "mean", n > 0, 4));
    OK_OR_RETURN(check_out(d_rstd, "rstd", n > 0, 4));
    mdl::GroupNormArgs a = group_norm_args(desc, packed(n, tokens, longest, d_offsets, d_order));
    const size_t need = mdl::groupnorm_workspace_bytes(a, false);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, need));
    OK_OR_RETURN(check_apart({span("y", d_y, tokens * cols * es, true), span("mean", d_mean, stats, true),
                              span("rstd", d_rstd, stats, true), span("the workspace", d_workspace, (int64_t)need, true),
                              span("x", d_x, rows_bytes(tokens, cols, x_stride, desc->dtype), false),
                              span("w", d_w, cols * 4, false), span("b", d_b, cols * 4, false),
                              span("offsets", d_offsets, ((int64_t)n + 1) * 8, false), span("order", d_order, (int64_t)n * 4, false)}));
    if (n == 0) return MDLSTM_OK;
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, need, stream));
    a.w = d_w;
    a.b = d_b;
    a.x = mdl::RowView{d_x, x_stride};
    a.y = d_y;
    a.mean = d_mean;
    a.rstd = d_rstd;
    a.ws = d_workspace;
    HIP_OR_FAIL(mdl::launch_groupnorm_fwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_group_norm_backward(const mdlstm_group_norm_desc* desc, int32_t n, int64_t tokens, int64_t longest,
                                         const int64_t* d_offsets, const int32_t* d_order, const void* d_x, int64_t x_stride,
                                         const float* d_w, const float* d_b, const float* d_mean, const float* d_rstd,
                                         const void* d_dy, int64_t dy_stride, void* d_dx, float* d_dw, float* d_db,
                                         void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_group_norm(desc));
    OK_OR_RETURN(check_sequences(n, tokens, longest));
    const int64_t cols = desc->channels, es = (int64_t)element(desc->dtype), stats = (int64_t)n * desc->groups * 4;
    OK_OR_RETURN(check_token_rows(d_x, "x", tokens, cols, x_stride, desc->dtype));
    OK_OR_RETURN(check_token_rows(d_dy, "dy", tokens, cols, dy_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_offsets, "offsets", n > 0, 8));
    OK_OR_RETURN(check_out(d_order, "order", false, 4));
    OK_OR_RETURN(check_out(d_w, "w", n > 0, 4));
    OK_OR_RETURN(check_out(d_b, "b", n > 0, 4));
    OK_OR_RETURN(check_out(d_mean, "mean", n > 0, 4));
    OK_OR_RETURN(check_out(d_rstd, "rstd", n > 0, 4));
    OK_OR_RETURN(check_out(d_dx, "dx", tokens > 0, es));
    OK_OR_RETURN(check_out(d_dw, "dw", true, 4));
    OK_OR_RETURN(check_out(d_db, "db", true, 4));
    mdl::GroupNormArgs a = group_norm_args(desc, packed(n, tokens, longest, d_offsets, d_order));
    const size_t need = mdl::groupnorm_workspace_bytes(a, true);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, need));
    OK_OR_RETURN(check_apart({span("dx", d_dx, tokens * cols * es, true), span("dw", d_dw, cols * 4, true),
                              span("db", d_db, cols * 4, true), span("the workspace", d_workspace, (int64_t)need, true),
                              span("x", d_x, rows_bytes(tokens, cols, x_stride, desc->dtype), false),
                              span("dy", d_dy, rows_bytes(tokens, cols, dy_stride, desc->dtype), false),
                              span("w", d_w, cols * 4, false), span("b", d_b, cols * 4, false), span("mean", d_mean, stats, false),
                              span("rstd", d_rstd, stats, false), span("offsets", d_offsets, ((int64_t)n + 1) * 8, false),
                              span("order", d_order, (int64_t)n * 4, false)}));
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, need, stream));
    a.w = d_w;
    a.b = d_b;
    a.x = mdl::RowView{d_x, x_stride};
    a.dy = mdl::RowView{d_dy, dy_stride};
    a.mean = const_cast<float*>(d_mean);
    a.rstd = const_cast<float*>(d_rstd);
    a.dx = d_dx;
    a.dw = d_dw;
    a.db = d_db;
    a.ws = d_workspace;
    HIP_OR_FAIL(mdl::launch_groupnorm_bwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

size_t mdlstm_vocabulary_workspace_bytes(const mdlstm_vocabulary_desc* desc, int64_t rows, int32_t backward) {
    if (check_vocabulary(desc, rows) != MDLSTM_OK) return 0;
    return mdl::vocabulary_workspace_bytes(vocabulary_args(desc, rows), backward != 0);
}

mdlstm_status mdlstm_vocabulary_forward(const mdlstm_vocabulary_desc* desc, int64_t rows, const void* d_x, int64_t x_stride,
                                        const void* d_w, int64_t w_stride, const int64_t* d_targets, float* d_losses,
                                        float* d_stats, void* d_workspace, size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_vocabulary(desc, rows));
    const int64_t dim = desc->dim;
    OK_OR_RETURN(check_rows(d_x, "x", rows, dim, x_stride, desc->dtype));
    OK_OR_RETURN(check_rows(d_w, "w", desc->vocab, dim, w_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_targets, "targets", rows > 0, 8));
    OK_OR_RETURN(check_out(d_losses, "losses", rows > 0, 4));
    OK_OR_RETURN(check_out(d_stats, "stats", rows > 0, 4));
    mdl::VocabularyArgs a = vocabulary_args(desc, rows);
    const size_t need = mdl::vocabulary_workspace_bytes(a, false);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, need));
    OK_OR_RETURN(check_apart({span("losses", d_losses, rows * 4, true), span("stats", d_stats, rows * 8, true),
                              span("the workspace", d_workspace, (int64_t)need, true),
                              span("x", d_x, rows_bytes(rows, dim, x_stride, desc->dtype), false),
                              span("w", d_w, rows_bytes(desc->vocab, dim, w_stride, desc->dtype), false),
                              span("targets", d_targets, rows * 8, false)}));
    if (rows == 0) return MDLSTM_OK;
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, need, stream));
    a.x = mdl::RowView{d_x, x_stride};
    a.w = mdl::RowView{d_w, w_stride};
    a.targets = d_targets;
    a.losses = d_losses;
    a.stats = d_stats;
    a.ws = d_workspace;
    HIP_OR_FAIL(mdl::launch_vocabulary_fwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

mdlstm_status mdlstm_vocabulary_backward(const mdlstm_vocabulary_desc* desc, int64_t rows, const void* d_x, int64_t x_stride,
                                         const void* d_w, int64_t w_stride, const int64_t* d_targets, const float* d_stats,
                                         const float* d_dlosses, void* d_dx, void* d_dw, void* d_workspace,
                                         size_t workspace_bytes, void* stream) {
    OK_OR_RETURN(check_vocabulary(desc, rows));
    const int64_t dim = desc->dim, es = (int64_t)element(desc->dtype);
    OK_OR_RETURN(check_rows(d_x, "x", rows, dim, x_stride, desc->dtype));
    OK_OR_RETURN(check_rows(d_w, "w", desc->vocab, dim, w_stride, desc->dtype));
    OK_OR_RETURN(check_out(d_targets, "targets", rows > 0, 8));
    OK_OR_RETURN(check_out(d_stats, "stats", rows > 0, 4));
    OK_OR_RETURN(check_out(d_dlosses, "dlosses", rows > 0, 4));
    OK_OR_RETURN(check_out(d_dx, "dx", rows > 0, es));
    OK_OR_RETURN(check_out(d_dw, "dw", true, es));
    mdl::VocabularyArgs a = vocabulary_args(desc, rows);
    const size_t need = mdl::vocabulary_workspace_bytes(a, true);
    OK_OR_RETURN(check_workspace(d_workspace, workspace_bytes, need));
    OK_OR_RETURN(check_apart({span("dx", d_dx, rows * dim * es, true), span("dw", d_dw, desc->vocab * dim * es, true),
                              span("the workspace", d_workspace, (int64_t)need, true),
                              span("x", d_x, rows_bytes(rows, dim, x_stride, desc->dtype), false),
                              span("w", d_w, rows_bytes(desc->vocab, dim, w_stride, desc->dtype), false),
                              span("targets", d_targets, rows * 8, false), span("stats", d_stats, rows * 8, false),
                              span("dlosses", d_dlosses, rows * 4, false)}));
    OK_OR_RETURN(mdl::poison_workspace(d_workspace, need, stream));
    a.x = mdl::RowView{d_x, x_stride};
    a.w = mdl::RowView{d_w, w_stride};
    a.targets = d_targets;
    a.stats = const_cast<float*>(d_stats);
    a.dloss = d_dlosses;
    a.dx = d_dx;
    a.dw = d_dw;
    a.ws = d_workspace;
    HIP_OR_FAIL(mdl::launch_vocabulary_bwd(a, reinterpret_cast<hipStream_t>(stream)));
    return MDLSTM_OK;
}

}  // extern "C"
